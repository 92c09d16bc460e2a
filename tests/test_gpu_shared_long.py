"""tkv_quant_attn_decode_shared over caches in which every wave goes through its ring of blocks many times and works its table of
token-independent terms out more than twice: all six settings with 16, 32 and 64 rows, long sequences of the batch's own beside a
prefix, numbers of blocks that divide unevenly; every KV head and sequence against float64 on the GPU.

Tolerance: that of the shorter cases (the framework's 2e-3 of a head's largest output; a block taken twice, left out or read with
another's scalers is off by far more: each row's weights lie mostly on one stretch of tokens)."""
import numpy as np
import pytest
import torch

import paper_2505_19586_amd as tkv
from oracle import quant

pytestmark = pytest.mark.gpu
SM = 128 ** -0.5
SETTINGS = [(1, 32), (1, 64), (2, 32), (2, 64), (4, 32), (4, 64)]


def _quantized(x, bits):
    """Eq. 4 along the last axis, dequantized in float64 (float32 steps as in the oracle)."""
    z = x.amin(-1, keepdim=True)
    s = ((x.amax(-1, keepdim=True).float() - z.float()) / (2 ** bits - 1)).half()
    code = torch.where(s == 0, 0.0, torch.round((x.float() - z.float()) / s.float()).clamp(0, 2 ** bits - 1))
    return code.double() * s.double() + z.double()


def _dequantized(k, v, bits, group, residual=128):
    """One head's rows [n, 128]."""
    nq = quant.partition(len(k), residual, group)[0]
    kq = _quantized(k[:nq].view(nq // group, group, 128).transpose(1, 2), bits).transpose(1, 2).reshape(nq, 128)
    vq = _quantized(v[:nq].view(nq, 128 // group, group), bits).reshape(nq, 128)
    return torch.cat([kq, k[nq:].double()]), torch.cat([vq, v[nq:].double()])


def _rows(batch, n, hkv, gen):
    """Keys with a direction that turns slowly along the tokens, so that a query looks at a stretch of them; values around 0.5."""
    k = torch.randn(batch, n, hkv, 128, generator=gen, device="cuda", dtype=torch.float16)
    t = torch.arange(n, device="cuda", dtype=torch.float32)
    for c in range(8):
        k[..., c] += (3 * torch.cos(t * (2 * np.pi / 40000) * (c + 1) + c)).half()[None, :, None]
    v = torch.randn(batch, n, hkv, 128, generator=gen, device="cuda", dtype=torch.float16)
    return k, v + 0.5


def _part(q, k, v):
    """Rows' largest logits, sums of exponentials and weighted values over one stretch of tokens (none: -inf, 0, 0)."""
    if len(k) == 0:
        return q.new_full((len(q), 1), -float("inf")), q.new_zeros(len(q), 1), q.new_zeros(len(q), 128)
    s = q @ k.T.contiguous() * SM
    m = s.amax(1, keepdim=True)
    w = torch.exp(s - m)
    return m, w.sum(1, keepdim=True), w @ v


def _check(out, q, prefix, own, lens, of, bits, group, hkv):
    """prefix, own: (k, v) [B, n, Hkv, 128]; of: every sequence's prefix, -1: none.  Each prefix once for all of its sequences."""
    grp, batch, worst = q.shape[1] // hkv, len(lens), 0.0
    for h in range(hkv):
        qs, got = (x[:, h * grp:(h + 1) * grp].double() for x in (q, out))
        shared = {}
        for i in set(of) - {-1}:
            of_it = [b for b in range(batch) if of[b] == i]
            m, l, o = _part(qs[of_it].reshape(-1, 128), *_dequantized(prefix[0][i, :, h], prefix[1][i, :, h], bits, group))
            shared.update({b: (m[y * grp:(y + 1) * grp], l[y * grp:(y + 1) * grp], o[y * grp:(y + 1) * grp]) for y, b in enumerate(of_it)})
        for b in range(batch):
            parts = [_part(qs[b], *_dequantized(own[0][b, :lens[b], h], own[1][b, :lens[b], h], bits, group))] + ([shared[b]] if of[b] >= 0 else [])
            top = torch.stack([m for m, _, _ in parts]).amax(0)
            total = sum(l * torch.exp(m - top) for m, l, _ in parts)
            ref = sum(o * torch.exp(m - top) for m, _, o in parts) / total
            worst = max(worst, float(((got[b] - ref).abs().amax(1) / ref.abs().amax(1)).max()))
    assert worst <= 2e-3, worst


def _layer(k, v, lens, hq, bits, group):
    L = tkv.QuantLayer(n_q_heads=hq, n_kv_heads=k.shape[2], bits=bits, group_size=group, capacity=(k.shape[1] + 63) // 64 * 64, batch=len(lens))
    L.append(k, v, n_valid=lens)
    return L


@pytest.mark.parametrize("bits,group", SETTINGS)
@pytest.mark.parametrize("hq,hkv,batch", [(64, 64, 12), (96, 32, 9), (96, 32, 16)])  # 12, 27 and 48 rows: 16, 32 and 64 at a time
def test_prefix(hq, hkv, batch, bits, group):
    # 256 workgroups of 8 waves: 256 / hkv chunks; 2 1/2 tables (of 8 or 16 groups) of blocks for every wave, and one block more
    blocks = 256 // hkv * 8 * (5 * (8 if bits == 4 else 16) * (group // 32) // 2) + 1
    n = 32 * blocks + 128 + (group // 2 + 3)
    print(f"case prefix {n} x {hkv} under {batch} x {hq // hkv}, {bits} bit/{group}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(bits * group + hq)
    k, v = _rows(1, n, hkv, gen)
    # the reference's quantizer is the oracle's
    c = quant.quantize_kv(k[0, :512, :1].transpose(0, 1).cpu().numpy(), v[0, :512, :1].transpose(0, 1).cpu().numpy(), bits=bits, group=group, residual=128)
    kd, vd = _dequantized(k[0, :512, 0], v[0, :512, 0], bits, group)
    assert np.array_equal(quant.dequantize_k(c)[0], kd[:c.n_quant].cpu().numpy()) and np.array_equal(quant.dequantize_v(c)[0], vd[:c.n_quant].cpu().numpy())
    own, lens = _rows(batch, 9, hkv, gen), [(4 * b) % 10 for b in range(batch)]
    P, L = _layer(k, v, [n], hq, bits, group), _layer(*own, lens, hq, bits, group)
    q = torch.randn(batch, hq, 128, generator=gen, device="cuda", dtype=torch.float16)
    plan = tkv.SharedPrefix(P, L)
    out = plan.attn_decode(q, SM)
    _check(out, q, (k, v), own, lens, [0] * batch, bits, group, hkv)
    assert torch.equal(out, plan.attn_decode(q, SM))


@pytest.mark.parametrize("bits,group", SETTINGS)
@pytest.mark.parametrize("hq,hkv,prefix_len", [(8, 8, 700), (64, 8, 20011)])  # 1 and 40 rows: their own tokens 16 rows at a time in either
def test_own_tokens(hq, hkv, prefix_len, bits, group):
    lens = [70001, 33, 40100, 5003, 0]
    print(f"case own {lens} over {prefix_len}, heads {hq}/{hkv}, {bits} bit/{group}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(bits * group + hq)
    prefix, own = _rows(2, prefix_len, hkv, gen), _rows(len(lens), max(lens), hkv, gen)
    P, L = _layer(*prefix, [prefix_len] * 2, hq, bits, group), _layer(*own, lens, hq, bits, group)
    q = torch.randn(len(lens), hq, 128, generator=gen, device="cuda", dtype=torch.float16)
    plan = tkv.SharedPrefix(P, L)
    for of in ([1] * 5, [0, -1, 1, 0, 1]):
        out = plan.attn_decode(q, SM, prefix_of=of)
        _check(out, q, prefix, own, lens, of, bits, group, hkv)
