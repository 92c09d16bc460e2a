"""Operators of a prompt's way into the cache and of a batch that shares one, each as `paper_2505_19586_amd` computes it and
in plain torch operations:

  rope    queries and keys normed per head and rotated in one pass, values laid out beside them (tkv.qk_norm_rope)
  prompt  attention over packed prompts: causal, grouped heads, chunks over earlier context, single tokens
          (tkv.PromptAttention)
  shared  decode attention of a batch whose sequences share long quantized prefixes, held and read once
          (tkv.SharedPrefix over two tkv.QuantLayer)

Head layouts and contexts are those of the repository's benchmark and tests: 32/8, 32/4, 64/8 and 32/32 heads of 128
channels, contexts up to 131072 tokens, caches of 1, 2 and 4 bits in groups of 32 or 64.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

D = 128
SM = 1.0 / math.sqrt(D)
DEV = "cuda:0"
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------------------------------------------------
# cases

def _rope(name, t, hq=32, hkv=8, src="fp16", dst="fp16", norm=True, interleaved=False, rot=128, pos0=0, values=True, fused=True):
    return {"name": name, "kind": "rope", "t": t, "hq": hq, "hkv": hkv, "src": src, "dst": dst, "norm": norm,
            "interleaved": interleaved, "rot": rot, "pos0": pos0, "values": values, "fused": fused}


def _prompt(name, n_q, n_k, batch=1, q_min=0, k_min=0, hq=32, hkv=8, dtype="fp16", causal=True):
    return {"name": name, "kind": "prompt", "batch": batch, "n_q": n_q, "n_k": n_k, "q_min": q_min or n_q,
            "k_min": k_min or n_k, "hq": hq, "hkv": hkv, "dtype": dtype, "causal": causal}


def _shared(name, n_prefix, batch, n_own, own_min=0, prefixes=1, bits=2, group=32, hq=32, hkv=8):
    return {"name": name, "kind": "shared", "n_prefix": n_prefix, "prefixes": prefixes, "batch": batch, "n_own": n_own,
            "own_min": own_min, "bits": bits, "group": group, "hq": hq, "hkv": hkv}


def listed():
    return [
        # one decode step of a small batch in a bfloat16 model whose caches hold fp16 rows: all latency
        _rope("rope_step_b16", 16, src="bf16", pos0=4000),
        # a whole 32k prompt in fp16, q, k, v as slices of the fused projection's rows
        _rope("rope_prompt_32k", 32768),
        # the last chunk of a long prompt in bfloat16, adjacent channels paired, half of the channels rotated, far positions,
        # an odd number of tokens, no values
        _rope("rope_chunk_odd", 10007, hkv=4, src="bf16", dst="bf16", interleaved=True, rot=64, pos0=121000, values=False, fused=False),
        # a prompt of ordinary length
        _prompt("prompt_4k", 4096, 4096),
        # the largest: a long prompt in one call
        _prompt("prompt_16k", 16384, 16384),
        # several prompts packed into one call, from one token to 4000, bfloat16, eight query heads per KV head
        _prompt("prompt_packed8", 4001, 4001, batch=8, q_min=1, k_min=1, hq=64, dtype="bf16"),
        # an odd last chunk of a prompt over what is cached already: few rows, many keys
        _prompt("prompt_chunk_64k", 333, 65536 + 333),
        # single tokens of four sequences over unquantized caches of different lengths
        _prompt("prompt_token_b4", 1, 32001, batch=4, q_min=1, k_min=9000, hkv=4),
        # a short system prompt under a small batch: all latency
        _shared("shared_2k_b4", 2000, 4, 300),
        # a 131072-token document under sixteen conversations, the benchmark's quantized layer
        _shared("shared_128k_b16", 131072, 16, 2000, own_min=1),
        # the method's own setting (1 bit, groups of 64, eight query heads per KV head), two prefixes of odd length
        _shared("shared_48k_1bit", 48413, 8, 4000, own_min=200, prefixes=2, bits=1, group=64, hkv=4),
        # the largest batch, 4 bits, eight query heads per KV head
        _shared("shared_32k_b64_4bit", 32770, 64, 500, bits=4, hq=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = ((32, 8), (32, 8), (32, 4), (64, 8), (32, 32))


def draw(rng):
    kind = rng.choices(("rope", "prompt", "shared"), (3, 5, 4))[0]
    hq, hkv = rng.choice(HEADS)
    if kind == "rope":
        src, dst = rng.choice((("fp16", "fp16"), ("bf16", "fp16"), ("bf16", "bf16"), ("fp16", "fp16")))
        return {"kind": kind, "t": _log_int(rng, 1, 32768 * 48 // (hq + 2 * hkv)), "hq": hq, "hkv": hkv, "src": src, "dst": dst,
                "norm": rng.random() < 0.7, "interleaved": rng.random() < 0.3, "rot": rng.choice((128, 128, 96, 64, 32)),
                "pos0": rng.choice((0, 0, 7, 60001, 130000)), "values": rng.random() < 0.6, "fused": rng.random() < 0.5}
    if kind == "prompt":
        batch = rng.choice((1, 1, 2, 4, 7, 16))
        causal = rng.random() < 0.85
        most = 16384 * 16384 * 32 // (hq * batch) // (1 if causal else 2)  # pairs of a padded sequence
        form = rng.choice(("whole", "whole", "chunk", "token"))
        if form == "whole":
            n_q = n_k = _log_int(rng, 1, min(16384, math.isqrt(most)))
            q_min = k_min = 1 if rng.random() < 0.5 else n_q
        else:
            n_q = 1 if form == "token" else _log_int(rng, 2, 1000)
            n_k = n_q + _log_int(rng, 1, min(100000 * 8 // (hkv * batch), most // n_q))
            q_min, k_min = max(1, n_q // 2), max(1, n_k // 3)
        return {"kind": kind, "batch": batch, "n_q": n_q, "n_k": n_k, "q_min": q_min, "k_min": k_min, "hq": hq, "hkv": hkv,
                "dtype": rng.choice(("fp16", "bf16")), "causal": causal}
    bits, group = rng.choice(((2, 32), (2, 32), (4, 32), (1, 64), (2, 64), (4, 64), (1, 32)))
    batch = rng.choice((1, 2, 3, 4, 8, 16, 32, 64))
    prefixes = rng.choice((1, 1, 1, 2)) if batch > 1 else 1
    n_prefix = _log_int(rng, 100, min(131072, 131072 * 8 // (hkv * prefixes), 64 * 64 * 32768 // (batch * hq)))
    n_own = _log_int(rng, 1, min(20000, 300000 // (batch * hkv)))
    return {"kind": kind, "n_prefix": n_prefix, "prefixes": prefixes, "batch": batch, "n_own": n_own,
            "own_min": rng.choice((0, n_own // 3, n_own)), "bits": bits, "group": group, "hq": hq, "hkv": hkv}


# ---------------------------------------------------------------------------------------------------------------------
# inputs

def _spread(batch, lo, hi):
    """Lengths of the sequences of a batch: the longest first, the others spread over [lo, hi]."""
    return [hi if b == 0 else lo + int((hi - lo) * ((b * 0.6180339887) % 1.0)) for b in range(batch)]


def _starts(lens):
    return [sum(lens[:b]) for b in range(len(lens))]


def _prompt_lens(case):
    q = _spread(case["batch"], case["q_min"], case["n_q"])
    k = _spread(case["batch"], case["k_min"], case["n_k"])
    return q, [max(a, b) for a, b in zip(q, k)]


def _randn(gen, *shape, dtype=torch.float16):
    return torch.randn(*shape, generator=gen, device=DEV, dtype=torch.float32).to(dtype)


def _rope_inputs(case, gen):
    t, hq, hkv, src = case["t"], case["hq"], case["hkv"], TYPES[case["src"]]
    heads = hq + 2 * hkv
    if case["fused"]:  # slices of one projection's rows
        rows = _randn(gen, t, heads, D, dtype=src)
        q, k, v = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
    else:
        q, k, v = (_randn(gen, t, h, D, dtype=src) for h in (hq, hkv, hkv))
    s = {"q": q, "k": k, "v": v if case["values"] else None, "q_weight": None, "k_weight": None}
    if case["norm"]:
        s["q_weight"], s["k_weight"] = ((1 + 0.2 * torch.randn(D, generator=gen, device=DEV)).to(src) for _ in range(2))
    s["positions"] = (case["pos0"] + torch.arange(t, device=DEV)).to(torch.int32)
    rot = case["rot"]
    s["inv_freq"] = (500000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)).float()
    return s


def _prompt_inputs(case, gen):
    q_lens, k_lens = _prompt_lens(case)
    dt = TYPES[case["dtype"]]
    q = _randn(gen, sum(q_lens), case["hq"], D, dtype=dt)
    k = _randn(gen, sum(k_lens), case["hkv"], D, dtype=dt)
    v = _randn(gen, sum(k_lens), case["hkv"], D, dtype=dt)
    k[:, :, torch.randperm(D, generator=gen, device=DEV)[:4]] *= 4  # key channels that stand out
    return {"q": q, "k": k, "v": v, "q_lens": q_lens, "k_lens": k_lens}


def _code_places(bits):
    """Word and field of code (t, c) of a block of 32 tokens x 128 channels: keys, values; int64 [32, 128] each."""
    t, c = torch.meshgrid(torch.arange(32, device=DEV), torch.arange(D, device=DEV), indexing="ij")
    lane = 4 * (t // 8) + t % 4 + 16 * ((c % 32) // 8)
    tau, v_lane = (t % 8) // 4, c % 16 + 16 * (t // 8)
    if bits == 1:
        return ((64 * tau + lane, (c % 8) // 2 + 4 * ((c // 32) % 2) + 8 * (c // 64) + 16 * (c % 2)),
                (64 * (c // 64) + v_lane, (t % 8) // 2 + 4 * ((c // 16) % 2) + 8 * ((c // 32) % 2) + 16 * (t % 2)))
    if bits == 2:
        return ((4 * lane + 2 * tau + c // 64, (c % 8) // 2 + 4 * ((c // 32) % 2) + 8 * (c % 2)),
                (4 * v_lane + c // 32, (t % 8) // 2 + 4 * ((c // 16) % 2) + 8 * (t % 2)))
    return ((256 * tau + 4 * lane + c // 32, (c % 8) // 2 + 4 * (c % 2)),
            (256 * (c // 64) + 4 * v_lane + (c // 16) % 4, (t % 8) // 2 + 4 * (t % 2)))


def _pack(codes, place, bits):
    """codes int32 [..., J, 32, 128] -> words int32 [..., J, 128 bits]."""
    fields = 32 // bits
    order = torch.empty(32 * D, dtype=torch.int64, device=DEV)
    order[(place[0] * fields + place[1]).reshape(-1)] = torch.arange(32 * D, device=DEV)
    by_word = codes.flatten(-2)[..., order].unflatten(-1, (-1, fields))
    return (by_word << (bits * torch.arange(fields, device=DEV, dtype=torch.int32))).sum(-1, dtype=torch.int32)


def _quantized(x, bits):
    """x [..., n] -> codes, scaler, zero-point of the groups along the last axis."""
    z = x.amin(-1)
    s = ((x.amax(-1).float() - z.float()) / (2 ** bits - 1)).half()
    code = torch.round((x.float() - z.float()[..., None]) / s.float()[..., None])
    return torch.where(s[..., None] == 0, 0, code).clamp(0, 2 ** bits - 1).to(torch.int32), s, z


def _cache(k, v, n, case, capacity):
    """The buffers of a quantized layer that holds n tokens (k, v fp16 [B, Hkv, capacity, 128]; n host ints)."""
    bits, g, w = case["bits"], case["group"], 128
    b, h, j = k.shape[0], k.shape[1], capacity // 32
    kp, vp = _code_places(bits)
    kc, ks, kz = _quantized(k.unflatten(2, (-1, g)).transpose(3, 4), bits)               # groups of g tokens, per channel
    k_words = _pack(kc.transpose(3, 4).reshape(b, h, j, 32, D), kp, bits)
    vc, vs, vz = _quantized(v.unflatten(3, (-1, g)), bits)                                # groups of g channels, per token
    v_words = _pack(vc.reshape(b, h, j, 32, D), vp, bits)
    meta = [x.unflatten(2, (j, 32)).transpose(3, 4).contiguous() for x in (vs, vz)]
    ring, nq = w + g, torch.tensor([(m - w) // g * g if m >= w else 0 for m in n], device=DEV)
    slot = torch.arange(ring, device=DEV)
    token = (nq[:, None] + (slot - nq[:, None]) % ring).clamp(max=capacity - 1)             # [B, ring]: the token at each slot
    at = token[:, None, :, None].expand(b, h, ring, D)
    return {"k_codes": k_words, "k_scale": ks, "k_zero": kz, "v_codes": v_words, "v_scale": meta[0], "v_zero": meta[1],
            "k_resid": k.gather(2, at), "v_resid": v.gather(2, at)}


def _lens_of(case):
    lens = _spread(case["batch"], case["own_min"], case["n_own"])
    prefix_lens = [case["n_prefix"] - 37 * p for p in range(case["prefixes"])]
    return prefix_lens, lens, [b * case["prefixes"] // case["batch"] for b in range(case["batch"])]


def _shared_inputs(case, gen):
    prefix_lens, lens, prefix_of = _lens_of(case)
    hq, hkv = case["hq"], case["hkv"]

    def rows(batch, capacity):
        k, v = (torch.randn(batch, hkv, capacity, D, generator=gen, device=DEV, dtype=torch.float16) for _ in range(2))
        k[..., :4] *= 4  # key channels that stand out
        return k, v

    caps = [(max(n) + 63) // 64 * 64 + 64 for n in (prefix_lens, lens)]
    s = {"q": _randn(gen, case["batch"], hq, D), "prefix_lens": prefix_lens, "lens": lens, "prefix_of": prefix_of, "caps": caps,
         "bits": case["bits"], "group": case["group"]}
    s["prefix"] = _cache(*rows(case["prefixes"], caps[0]), prefix_lens, case, caps[0])
    s["cache"] = _cache(*rows(case["batch"], caps[1]), lens, case, caps[1])
    return s


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    s = {"rope": _rope_inputs, "prompt": _prompt_inputs, "shared": _shared_inputs}[case["kind"]](case, gen)
    s["case"] = case
    if own:
        import paper_2505_19586_amd as tkv

        s["tkv"] = tkv
        if case["kind"] == "prompt":
            s["plan"] = tkv.PromptAttention(n_q_heads=case["hq"], n_kv_heads=case["hkv"], dtype=TYPES[case["dtype"]],
                                            causal=case["causal"], batch=case["batch"])
        if case["kind"] == "shared":
            both = []
            for name, n, cap in (("prefix", s["prefix_lens"], s["caps"][0]), ("cache", s["lens"], s["caps"][1])):
                layer = tkv.QuantLayer(n_q_heads=case["hq"], n_kv_heads=case["hkv"], bits=case["bits"], group_size=case["group"],
                                       capacity=cap, batch=len(n))
                for key, x in s.pop(name).items():
                    layer.buffers[key][:x.nbytes].copy_(x.contiguous().view(-1).view(torch.uint8))
                layer.seq_len[:] = n
                both.append(layer)
            s["plan"] = tkv.SharedPrefix(*both)
            s["prefix_of"] = np.array(s["prefix_of"], dtype=np.int32)
    return s


# ---------------------------------------------------------------------------------------------------------------------
# one pass

def _plain_rope(s):
    case, dst = s["case"], TYPES[s["case"]["dst"]]
    rot = case["rot"]
    angle = s["positions"].double()[:, None] * s["inv_freq"].double()  # 64 bits: far positions
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def turned(x, weight):
        x = x.float()
        if weight is not None:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * weight.float()
        y, rest = x[..., :rot], x[..., rot:]
        if case["interleaved"]:
            a, b = y[..., 0::2], y[..., 1::2]
            y = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
        else:
            a, b = y[..., :rot // 2], y[..., rot // 2:]
            y = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
        return torch.cat((y, rest), -1).to(dst)

    out = {"q": turned(s["q"], s["q_weight"]), "k": turned(s["k"], s["k_weight"])}
    if s["v"] is not None:
        out["v"] = s["v"].to(dst).contiguous()
    return out


def _padded(x, lens):
    """Packed rows [T, H, D] -> float32 [B, H, longest, D]."""
    n = torch.tensor(lens, device=x.device)
    at = torch.arange(max(lens), device=x.device)
    rows = (torch.tensor(_starts(lens), device=x.device)[:, None] + at).clamp(max=x.shape[0] - 1)
    return torch.where((at < n[:, None])[..., None, None], x[rows].float(), 0).transpose(1, 2)


def _plain_prompt(s):
    case, q_lens, k_lens = s["case"], s["q_lens"], s["k_lens"]
    b, g = case["batch"], case["hq"] // case["hkv"]
    q, k, v = _padded(s["q"], q_lens), _padded(s["k"], k_lens), _padded(s["v"], k_lens)
    nq, nk = (torch.tensor(n, device=q.device)[:, None, None] for n in (q_lens, k_lens))
    i, j = torch.arange(q.shape[2], device=q.device)[:, None], torch.arange(k.shape[2], device=q.device)
    seen = (j < nk) & (j <= i + nk - nq) if case["causal"] else (j < nk).expand(b, q.shape[2], -1)
    w = torch.matmul(q.unflatten(1, (-1, g)).flatten(2, 3) * SM, k.transpose(2, 3)).unflatten(2, (g, -1))  # [B, Hkv, G, Q, K]
    w = w.masked_fill_(~seen[:, None, None], -math.inf)
    top = w.amax(-1, keepdim=True)
    w = w.sub_(top).exp_()
    total = w.sum(-1, keepdim=True)
    out = torch.matmul(w.flatten(2, 3), v).unflatten(2, (g, -1)) / total
    lse = (top + total.log()).squeeze(-1)
    real = torch.arange(q.shape[2], device=q.device) < torch.tensor(q_lens, device=q.device)[:, None]  # [B, Q]
    return {"out": out.flatten(1, 2).transpose(1, 2)[real].to(s["q"].dtype), "lse": lse.flatten(1, 2).transpose(1, 2)[real]}


def _plain_rows(cache, lens, bits, g):
    """A cache's keys and values in float32 [B, Hkv, longest, 128]."""
    longest, ring = max(lens), cache["k_resid"].shape[2]
    kp, vp = _code_places(bits)
    mask = 2 ** bits - 1
    blocks = -(-longest // 64) * 2
    kc = (cache["k_codes"][:, :, :blocks, kp[0]] >> (bits * kp[1]).to(torch.int32)) & mask  # [B, Hkv, J, 32, 128]
    vc = (cache["v_codes"][:, :, :blocks, vp[0]] >> (bits * vp[1]).to(torch.int32)) & mask
    groups = blocks * 32 // g
    k = kc.flatten(2, 3).unflatten(2, (groups, g)) * cache["k_scale"][:, :, :groups, None].float() + cache["k_zero"][:, :, :groups, None].float()
    vs, vz = (cache[n][:, :, :blocks].transpose(3, 4).float()[..., None] for n in ("v_scale", "v_zero"))  # [B, Hkv, J, 32, 128 / g, 1]
    v = vc.unflatten(4, (-1, g)) * vs + vz
    t = torch.arange(longest, device=DEV)
    nq = torch.tensor([(m - 128) // g * g if m >= 128 else 0 for m in lens], device=DEV)
    coded = (t < nq[:, None])[:, None, :, None]
    return [torch.where(coded, x[:, :, :longest], cache[r][:, :, t % ring].float())
            for x, r in ((k.flatten(2, 3), "k_resid"), (v.flatten(4, 5).flatten(2, 3), "v_resid"))]


def _plain_shared(s):
    q, bits, g = s["q"].float() * SM, s["bits"], s["group"]
    pk, pv = _plain_rows(s["prefix"], s["prefix_lens"], bits, g)  # [P, Hkv, Np, 128]
    ok, ov = _plain_rows(s["cache"], s["lens"], bits, g) if max(s["lens"]) else (torch.zeros(q.shape[0], pk.shape[1], 1, D, device=DEV),) * 2
    q = q.unflatten(1, (pk.shape[1], -1))  # [B, Hkv, G, 128]
    b, h, grp = q.shape[:3]
    np_, no = torch.tensor(s["prefix_lens"], device=DEV), torch.tensor(s["lens"], device=DEV)
    of, t = torch.tensor(s["prefix_of"], device=DEV), torch.arange(pk.shape[2], device=DEV)
    mine = (of[:, None] == torch.arange(len(s["prefix_lens"]), device=DEV))[:, :, None] & (t < np_[:, None])  # [B, P, Np]
    flat = q.transpose(0, 1).flatten(1, 2)  # [Hkv, B G, 128]
    wp = torch.matmul(flat, pk.transpose(2, 3)).unflatten(2, (b, grp))  # [P, Hkv, B, G, Np]
    wp = wp.masked_fill_(~mine.transpose(0, 1)[:, None, :, None], -math.inf)
    wo = torch.matmul(q, ok.transpose(2, 3)).masked_fill_((torch.arange(ok.shape[2], device=DEV) >= no[:, None])[:, None, None], -math.inf)
    top = torch.maximum(wp.amax((0, 4)).transpose(0, 1), wo.amax(-1))  # [B, Hkv, G]
    wp = wp.sub_(top.transpose(0, 1)[None, ..., None]).exp_()
    wo = wo.sub_(top[..., None]).exp_()
    total = wp.sum((0, 4)).transpose(0, 1) + wo.sum(-1)
    out = torch.matmul(wp.flatten(2, 3), pv).sum(0).unflatten(1, (b, grp)).transpose(0, 1) + torch.matmul(wo, ov)
    return {"out": (out / total[..., None]).flatten(1, 2).half()}


def run(state):
    s, case = state, state["case"]
    if not own:
        return {"rope": _plain_rope, "prompt": _plain_prompt, "shared": _plain_shared}[case["kind"]](s)
    if case["kind"] == "rope":
        q, k, v = s["tkv"].qk_norm_rope(s["q"], s["k"], s["positions"], s["inv_freq"], v=s["v"], norm=case["norm"],
                                        q_weight=s["q_weight"], k_weight=s["k_weight"], eps=1e-6,
                                        interleaved=case["interleaved"], out_dtype=TYPES[case["dst"]])
        return {"q": q, "k": k} if v is None else {"q": q, "k": k, "v": v}
    if case["kind"] == "prompt":
        out, lse = s["plan"].attend(s["q"], s["k"], s["v"], SM, s["q_lens"], s["k_lens"], lse=True)
        return {"out": out, "lse": lse}
    return {"out": s["plan"].attn_decode(s["q"], SM, prefix_of=s["prefix_of"])}


# ---------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without

def work(case):
    hq, hkv = case["hq"], case["hkv"]
    if case["kind"] == "rope":
        heads = hq + hkv + (hkv if case["values"] else 0)
        return {"bytes": case["t"] * (heads * D * 4 + 4) + 2 * case["rot"], "flops": case["t"] * (hq + hkv) * D * (7 if case["norm"] else 3)}
    if case["kind"] == "prompt":
        q_lens, k_lens = _prompt_lens(case)
        pairs = sum(a * b - a * (a - 1) // 2 if case["causal"] else a * b for a, b in zip(q_lens, k_lens))
        return {"bytes": sum(q_lens) * hq * (D * 4 + 4) + sum(k_lens) * hkv * D * 4, "flops": 4 * D * hq * pairs}
    prefix_lens, lens, of = _lens_of(case)
    size = 0
    for n in prefix_lens + lens:
        nq = (n - 128) // case["group"] * case["group"] if n >= 128 else 0
        size += hkv * (nq * (D * case["bits"] // 4 + 1024 // case["group"]) + (n - nq) * D * 4)
    tokens = sum(lens) + sum(prefix_lens[p] for p in of)
    return {"bytes": size + case["batch"] * hq * D * 4, "flops": 4 * D * hq * tokens}


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits

def _exact_rope(case, s):
    rot, half = case["rot"], case["rot"] // 2
    first = [2 * i if case["interleaved"] else i for i in range(half)]
    second = [2 * i + 1 if case["interleaved"] else i + half for i in range(half)]
    theta = torch.outer(s["positions"].double(), s["inv_freq"].double())
    turn = torch.polar(torch.ones_like(theta), theta)  # [T, half]
    out = {}
    for name, weight in (("q", s["q_weight"]), ("k", s["k_weight"])):
        x = s[name].double()
        if weight is not None:
            x = weight.double() * x / ((x * x).sum(2, keepdim=True) / D + 1e-6).sqrt()
        z = torch.complex(x[:, :, first], x[:, :, second]) * turn[:, None, :]
        y = x.clone()
        y[:, :, first], y[:, :, second] = z.real, z.imag
        out[name] = y
    if s["v"] is not None:
        out["v"] = s["v"].double()
    return out


def _exact_prompt(case, s):
    grp = case["hq"] // case["hkv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    q0 = k0 = 0
    for nq, nk in zip(s["q_lens"], s["k_lens"]):
        for h in range(case["hq"]):
            k, v = s["k"][k0:k0 + nk, h // grp].double(), s["v"][k0:k0 + nk, h // grp].double()
            for a in range(0, nq, 4096):
                q = s["q"][q0 + a:q0 + min(nq, a + 4096), h].double()
                logits = q @ k.T.contiguous() * SM
                if case["causal"]:
                    logits += torch.full_like(logits, -math.inf).triu(nk - nq + a + 1)
                at = slice(q0 + a, q0 + a + q.shape[0])
                lse[at, h] = torch.logsumexp(logits, 1)
                out[at, h] = torch.softmax(logits, 1) @ v
        q0, k0 = q0 + nq, k0 + nk
    return {"out": out, "lse": lse}


def _exact_places(bits):
    """(word, field) of key and value code (t, c), as the cache's documentation has them."""
    k, v = np.zeros((32, D, 2), np.int64), np.zeros((32, D, 2), np.int64)
    for t in range(32):
        for c in range(D):
            r, tau = 4 * (t // 8) + t % 4, t % 8 // 4
            lk, lv = r + 16 * (c % 32 // 8), c % 16 + 16 * (t // 8)
            if bits == 1:
                k[t, c] = 64 * tau + lk, c % 8 // 2 + 4 * (c // 32 % 2) + 8 * (c // 64) + 16 * (c % 2)
                v[t, c] = 64 * (c // 64) + lv, t % 8 // 2 + 4 * (c // 16 % 2) + 8 * (c // 32 % 2) + 16 * (t % 2)
            elif bits == 2:
                k[t, c] = 4 * lk + 2 * tau + c // 64, c % 8 // 2 + 4 * (c // 32 % 2) + 8 * (c % 2)
                v[t, c] = 4 * lv + c // 32, t % 8 // 2 + 4 * (c // 16 % 2) + 8 * (t % 2)
            else:
                k[t, c] = 256 * tau + 4 * lk + c // 32, c % 8 // 2 + 4 * (c % 2)
                v[t, c] = 256 * (c // 64) + 4 * lv + c // 16 % 4, t % 8 // 2 + 4 * (t % 2)
    return torch.from_numpy(k).to(DEV), torch.from_numpy(v).to(DEV)


def _exact_rows(cache, b, h, n, bits, g):
    """Keys and values of one sequence and KV head, float64 [n, 128] each."""
    nq = (n - 128) // g * g if n >= 128 else 0
    blocks, parts = nq // 32, []
    for name, place in zip("kv", _exact_places(bits)):
        words = cache[name + "_codes"][b, h, :blocks].long() & 0xFFFFFFFF
        code = ((words[:, place[..., 0].reshape(-1)] >> (bits * place[..., 1].reshape(-1))) % 2 ** bits).reshape(nq, D).double()
        scale, zero = cache[name + "_scale"][b, h].double(), cache[name + "_zero"][b, h].double()
        if name == "k":
            scale, zero = (x[:nq // g].repeat_interleave(g, 0) for x in (scale, zero))
        else:
            scale, zero = (x[:blocks].permute(0, 2, 1).reshape(nq, D // g).repeat_interleave(g, 1) for x in (scale, zero))
        tail = cache[name + "_resid"][b, h][torch.arange(nq, n, device=DEV) % (128 + g)].double()
        parts.append(torch.cat((code * scale + zero, tail)))
    return parts


def _exact_shared(case, s):
    grp = case["hq"] // case["hkv"]
    out = torch.zeros(case["batch"], case["hq"], D, dtype=torch.float64, device=DEV)
    for h in range(case["hkv"]):
        before = [_exact_rows(s["prefix"], p, h, n, case["bits"], case["group"]) for p, n in enumerate(s["prefix_lens"])]
        for b, n in enumerate(s["lens"]):
            k, v = (torch.cat(x) for x in zip(before[s["prefix_of"][b]], _exact_rows(s["cache"], b, h, n, case["bits"], case["group"])))
            heads = slice(h * grp, (h + 1) * grp)
            out[b, heads] = torch.softmax(s["q"][b, heads].double() @ k.T.contiguous() * SM, 1) @ v
    return {"out": out}


def exact(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    kind = case["kind"]
    s = {"rope": _rope_inputs, "prompt": _prompt_inputs, "shared": _shared_inputs}[kind](case, gen)
    return {"rope": _exact_rope, "prompt": _exact_prompt, "shared": _exact_shared}[kind](case, s)
