"""tkv_quant_attn_decode_shared against float64 over the dequantized prefix and own tokens: all six settings, head groups, batches
from one sequence to 64, prefixes of any length, none and several, rings that wrap, what lies behind the last token, streams,
replayed graphs and a run from a prompt's rows to shared decoding.

Tolerance: the framework's measure of attention outputs (max over heads of max_c |o - ref| / max_c |ref|) and its bound
of 2e-3: weights and outputs are fp16 numbers, off by at most 2^-11 = 4.9e-4 of each; codes, scalers and zero-points enter the
products unrounded, sums are float32."""
import numpy as np
import pytest
import torch

import paper_2505_19586_amd as tkv
from oracle import attention, quant
from oracle.prompt import prompt_attention
from oracle.rope import norm_rope
from synth import make_layer
from synth.workloads import HeadShape

from gpu_util import attn_err, to_new_batch

pytestmark = pytest.mark.gpu
SM = 128 ** -0.5
SETTINGS = [(1, 32), (1, 64), (2, 32), (2, 64), (4, 32), (4, 64)]


def _draw(n, hq, hkv, layer, seq):
    return make_layer(n, config=7, layer=layer, seq=seq, shape=HeadShape(hq, hkv, 128))


def _fill(lens, hq, hkv, bits, group, residual, layer, capacity=None):
    inps = [_draw(n, hq, hkv, layer, s) for s, n in enumerate(lens)]
    cap = capacity or (max(max(lens), 1) + 63) // 64 * 64
    L = tkv.QuantLayer(n_q_heads=hq, n_kv_heads=hkv, bits=bits, group_size=group, residual=residual, capacity=cap, batch=len(lens))
    if max(lens):
        L.append(to_new_batch([i.k for i in inps], max(lens)), to_new_batch([i.v for i in inps], max(lens)), n_valid=lens)
    return L, inps


def _rows(inp, bits, group, residual):
    c = quant.quantize_kv(inp.k, inp.v, bits=bits, group=group, residual=residual)
    return (np.concatenate([quant.dequantize_k(c), c.k_resid.astype(np.float64)], axis=1),
            np.concatenate([quant.dequantize_v(c), c.v_resid.astype(np.float64)], axis=1))


def _check(out, q, prefixes, owns, of):
    q = q.cpu().numpy()
    for b, (k, v) in enumerate(owns):
        if of[b] >= 0:
            k, v = (np.concatenate([x, y], axis=1) for x, y in zip(prefixes[of[b]], (k, v)))
        ref = attention.decode_attention(q[b], k, v, SM)
        if k.shape[1] == 0:
            assert (out[b] == 0).all()
        else:
            assert attn_err(out[b], ref) <= 2e-3, (b, attn_err(out[b], ref))


def _case(prefix_lens, lens, of=None, hq=8, hkv=2, bits=2, group=32, residuals=(128, 128), times=2):
    print(f"case prefixes {prefix_lens} own {lens} of {of} heads {hq}/{hkv} {bits} bit/{group}", flush=True)
    P, pi = _fill(prefix_lens, hq, hkv, bits, group, residuals[0], 1)
    L, oi = _fill(lens, hq, hkv, bits, group, residuals[1], 2)
    q = torch.from_numpy(np.stack([i.q for i in oi])).cuda()
    plan = tkv.SharedPrefix(P, L)
    out = plan.attn_decode(q, SM, prefix_of=of)
    torch.cuda.synchronize()
    _check(out, q, [_rows(i, bits, group, residuals[0]) for i in pi], [_rows(i, bits, group, residuals[1]) for i in oi],
           [0] * len(lens) if of is None else of)
    for _ in range(times - 1):
        plan.workspace.fill_(0xFF)      # NaN everywhere: nothing of it is read before it is written
        assert torch.equal(out, plan.attn_decode(q, SM, prefix_of=of))
    return plan, q, out


@pytest.mark.parametrize("bits,group", SETTINGS)
def test_settings(bits, group):
    _case([1000], [70, 300, 1, 0, 517], bits=bits, group=group)


@pytest.mark.parametrize("n", [1, 31, 32, 33, 127, 128, 159, 160, 161, 255, 256, 300, 700, 2049])
def test_prefix_lengths(n):
    _case([n], [3, 0, 200], bits=2, group=32)
    _case([n], [0, 0, 1], bits=1, group=64)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (5, 1), (8, 1), (14, 2), (32, 8)])
@pytest.mark.parametrize("batch", [1, 3, 9])
def test_heads_and_batches(hq, hkv, batch):
    _case([600], [(53 * b) % 170 for b in range(batch)], hq=hq, hkv=hkv, bits=4, group=32)


def test_largest_batch_and_groups():
    _case([900], [(7 * b) % 90 for b in range(64)], hq=8, hkv=1, bits=2, group=32)


def test_several_prefixes_and_none():
    _case([400, 0, 150, 700], [10, 200, 0, 33, 0, 5, 180], of=[3, -1, 0, 1, 1, 3, -1])
    _case([400, 300], [0, 0, 0], of=[-1, -1, -1])
    _case([64, 300], [0, 40], of=[1, 1], hq=8, hkv=8, bits=4, group=64)


def test_other_residuals():
    _case([1500], [600, 40], residuals=(64, 256))
    _case([1500], [1100, 40], residuals=(960, 64), bits=1, group=64)


def test_rings_that_have_wrapped_and_what_is_behind_the_last_token():
    """Caches grown token by token, so that the rings wrap; the slots behind the last token hold NaN before."""
    print("case wrapped rings", flush=True)
    hq, hkv = 8, 2
    P, L = (tkv.QuantLayer(n_q_heads=hq, n_kv_heads=hkv, bits=2, capacity=1024, batch=b) for b in (1, 2))
    for x in (P, L):
        for name in ("k_resid", "v_resid"):
            x.view(name).fill_(float("nan"))
    inps = [_draw(560, hq, hkv, 3, s) for s in range(3)]
    k, v = to_new_batch([i.k for i in inps], 560), to_new_batch([i.v for i in inps], 560)
    for a, b in ((0, 300), (300, 301), (301, 350), (350, 421)):
        P.append(k[:1, a:b].contiguous(), v[:1, a:b].contiguous())
    for a, b in ((0, 5), (5, 170), (170, 400), (400, 401), (401, 560)):
        L.append(k[1:, a:b].contiguous(), v[1:, a:b].contiguous(), n_valid=[b - a, b - a if b < 500 else 3])
    q = torch.from_numpy(np.stack([i.q for i in inps[1:]])).cuda()
    out = tkv.SharedPrefix(P, L).attn_decode(q, SM)
    torch.cuda.synchronize()

    def rows(i, n):
        c = quant.quantize_kv(inps[i].k[:, :n], inps[i].v[:, :n], bits=2, group=32, residual=128)
        return (np.concatenate([quant.dequantize_k(c), c.k_resid.astype(np.float64)], axis=1),
                np.concatenate([quant.dequantize_v(c), c.v_resid.astype(np.float64)], axis=1))

    _check(out, q, [rows(0, 421)], [rows(1, 560), rows(2, 404)], [0, 0])


def test_large_values_and_flat_groups():
    """Values up to 30000, groups of one value (scaler 0), one token that outweighs all others by far."""
    print("case large values", flush=True)
    hq, hkv, n = 4, 1, 700
    inp = _draw(n, hq, hkv, 4, 0)
    inp.v[:, ::7] = 30000
    inp.v[:, 3::7] = -30000
    inp.k[:, 64:128, :64] = 2
    inp.v[:, 32:64] = 1
    inp.k[0, 200] = 12 * inp.q[0]
    P = tkv.QuantLayer(n_q_heads=hq, n_kv_heads=hkv, bits=4, group_size=32, capacity=704)
    P.append(to_new_batch([inp.k], n), to_new_batch([inp.v], n))
    L, oi = _fill([60], hq, hkv, 4, 32, 128, 5)
    q = torch.from_numpy(inp.q)[None].cuda()
    out = tkv.SharedPrefix(P, L).attn_decode(q, SM)
    torch.cuda.synchronize()
    # (one logit of about 130 x 12 is off by 2^-12 of that at most)
    _check(out, q, [_rows(inp, 4, 32, 128)], [_rows(oi[0], 4, 32, 128)], [0])


def test_agrees_with_the_undivided_cache():
    """A prefix whose length is a multiple of the group plus the residual, no own tokens: the same cache as tkv_quant_attn_decode's."""
    plan, q, out = _case([32 * 40 + 128], [0, 0, 0, 0], hq=32, hkv=8)
    P = plan.prefix
    for b in range(4):
        alone = P.attn_decode(q[b:b + 1].contiguous(), SM)
        assert attn_err(out[b], alone[0].double().cpu().numpy()) <= 2e-3


def test_side_stream_and_replayed_graph():
    plan, q, want = _case([2000], [300, 10, 77], hq=32, hkv=8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = plan.attn_decode(q, SM)
    torch.cuda.synchronize()
    assert torch.equal(want, got)
    graph, out = torch.cuda.CUDAGraph(), torch.empty_like(q)
    with torch.cuda.graph(graph):
        plan.attn_decode(q, SM, out=out)
    for _ in range(4):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, plan.attn_decode(q, SM))
        q *= 0.75


def test_one_layer_as_prefix_and_batch_and_two_plans_at_once():
    """A layer may continue itself; two plans (a workspace each) run on two streams at the same time."""
    print("case same layer, two streams", flush=True)
    L, inps = _fill([500, 90], 8, 2, 2, 32, 128, 5)
    rows = [_rows(i, 2, 32, 128) for i in inps]
    q = torch.from_numpy(np.stack([i.q for i in inps])).cuda()
    plans = [tkv.SharedPrefix(L, L) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = [[p.attn_decode(q, SM, prefix_of=of, stream=s) for p, s, of in zip(plans, streams, ([1, 0], [-1, 1]))] for _ in range(8)]
    torch.cuda.synchronize()
    for a, b in outs:
        _check(a, q, rows, rows, [1, 0])
        _check(b, q, rows, rows, [-1, 1])
        assert torch.equal(a, outs[0][0]) and torch.equal(b, outs[0][1])


@pytest.mark.parametrize("bits,group,hq,hkv,batch,n", [(2, 32, 32, 8, 16, 131072), (1, 64, 64, 8, 40, 40001)])
def test_long_prefixes(bits, group, hq, hkv, batch, n):
    """Long prefixes against float64 on the GPU, of rows drawn there; values centred and not."""
    print(f"case long prefix {n} x {batch}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(n)
    k, v = (torch.randn(1, n, hkv, 128, generator=g, device="cuda", dtype=torch.float16) for _ in range(2))
    v += 0.5
    P = tkv.QuantLayer(n_q_heads=hq, n_kv_heads=hkv, bits=bits, group_size=group, capacity=(n + 63) // 64 * 64)
    P.append(k, v)
    L = tkv.QuantLayer(n_q_heads=hq, n_kv_heads=hkv, bits=bits, group_size=group, capacity=64, batch=batch)
    ko, vo = (torch.randn(batch, 9, hkv, 128, generator=g, device="cuda", dtype=torch.float16) for _ in range(2))
    L.append(ko, vo)
    q = torch.randn(batch, hq, 128, generator=g, device="cuda", dtype=torch.float16)
    out = tkv.SharedPrefix(P, L).attn_decode(q, SM)
    torch.cuda.synchronize()
    h = 3
    c = quant.quantize_kv(k[0, :, h:h + 1].transpose(0, 1).contiguous().cpu().numpy(), v[0, :, h:h + 1].transpose(0, 1).contiguous().cpu().numpy(),
                          bits=bits, group=group, residual=128)
    kk = np.concatenate([quant.dequantize_k(c), c.k_resid.astype(np.float64)], axis=1)[0]
    vv = np.concatenate([quant.dequantize_v(c), c.v_resid.astype(np.float64)], axis=1)[0]
    grp = hq // hkv
    for b in (0, batch // 2, batch - 1):
        ref = attention.decode_attention(q[b, h * grp:(h + 1) * grp].cpu().numpy(),
                                         np.concatenate([kk, ko[b, :, h].double().cpu().numpy()])[None],
                                         np.concatenate([vv, vo[b, :, h].double().cpu().numpy()])[None], SM)
        assert attn_err(out[b, h * grp:(h + 1) * grp], ref) <= 2e-3


def test_from_a_prompt_to_shared_decoding():
    """The operators one after the other: a bf16 model's rows normed and rotated into fp16, attention over the prompt,
    the prompt appended once, two conversations' tokens appended and attended over the shared prefix."""
    print("case prompt to decode", flush=True)
    hq, hkv, n, batch, own = 8, 2, 333, 2, 5
    g = torch.Generator(device="cuda").manual_seed(1)
    f = (500000.0 ** (-torch.arange(0, 128, 2, dtype=torch.float64) / 128)).float().cuda()
    qw, kw = ((1 + 0.2 * torch.randn(128, generator=g, device="cuda")).bfloat16() for _ in range(2))

    def rows(t, pos):
        x = torch.randn(t, hq + 2 * hkv, 128, generator=g, device="cuda").bfloat16()
        q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
        got = tkv.qk_norm_rope(q, k, pos, f, v=v, norm=True, q_weight=qw, k_weight=kw, out_dtype=torch.float16)
        a = dict(norm=True, eps=1e-6)
        want = [norm_rope(y.double().cpu().numpy(), pos.cpu().numpy(), f.cpu().numpy(), weight=w.double().cpu().numpy(), **a)[0]
                for y, w in ((q, qw), (k, kw))] + [v.double().cpu().numpy()]
        for o, w in zip(got, want):
            # half a step of fp16 and float32's errors
            assert np.abs(o.double().cpu().numpy() - w).max() <= 2.0 ** -11 * np.abs(w).max() + 2.0 ** -17
        return got

    q, k, v = rows(n, torch.arange(n, device="cuda", dtype=torch.int32))
    out = tkv.PromptAttention(n_q_heads=hq, n_kv_heads=hkv).attend(q, k, v, SM, [n])
    ref, _ = prompt_attention(q.cpu().numpy(), k.cpu().numpy(), v.cpu().numpy(), SM)
    assert np.abs(out.double().cpu().numpy() - ref).max() <= 2.1 * 2.0 ** -11 * np.abs(v.double().cpu().numpy()).max()
    P = tkv.QuantLayer(n_q_heads=hq, n_kv_heads=hkv, bits=4, capacity=352)
    P.append(k[None], v[None])
    L = tkv.QuantLayer(n_q_heads=hq, n_kv_heads=hkv, bits=4, capacity=64, batch=batch)
    plan = tkv.SharedPrefix(P, L)
    c = quant.quantize_kv(k.transpose(0, 1).contiguous().cpu().numpy(), v.transpose(0, 1).contiguous().cpu().numpy(), bits=4, group=32, residual=128)
    pk, pv = (np.concatenate(x, axis=1) for x in ((quant.dequantize_k(c), c.k_resid.astype(np.float64)), (quant.dequantize_v(c), c.v_resid.astype(np.float64))))
    ks, vs = [], []
    for step in range(own):
        q1, k1, v1 = rows(batch, torch.full((batch,), n + step, device="cuda", dtype=torch.int32))
        L.append(k1[:, None], v1[:, None])
        ks.append(k1.double().cpu().numpy())
        vs.append(v1.double().cpu().numpy())
        out = plan.attn_decode(q1, SM)
        for b in range(batch):
            ok, ov = (np.stack([x[b] for x in y], axis=1) for y in (ks, vs))
            ref = attention.decode_attention(q1[b].cpu().numpy(), np.concatenate([pk, ok], axis=1), np.concatenate([pv, ov], axis=1), SM)
            assert attn_err(out[b], ref) <= 2e-3
