"""tkv_quant_attn_decode_shared multiplies codes, scalers and zero-points without a rounding before its float32 sums: caches whose
dequantized rows nearly cancel, so that a rounding of theirs to fp16, or the lower bits of a scaler left out, would show.

Every product is a multiple of 2^-5 and every sum of them below 2^19 (of values with weights: of 2^-2, below 2^22), so that float32
holds them exactly, in any order.  What is left is named in each test."""
import numpy as np
import pytest
import torch

import paper_2505_19586_amd as tkv
from oracle import attention, quant

from gpu_util import to_new

pytestmark = pytest.mark.gpu
SM = 128 ** -0.5
SETTINGS = [(1, 32), (1, 64), (2, 32), (2, 64), (4, 32), (4, 64)]
BATCHES = [1, 5, 9]  # of eight query heads per KV head: 8, 40 and 72 rows


def _layers(k, v, bits, group, batch):
    """All tokens in the prefix, none of the sequences' own; the oracle's rows in float64."""
    P = tkv.QuantLayer(n_q_heads=16, n_kv_heads=2, bits=bits, group_size=group, residual=group, capacity=(k.shape[1] + 63) // 64 * 64)
    P.append(to_new(k), to_new(v))
    L = tkv.QuantLayer(n_q_heads=16, n_kv_heads=2, bits=bits, group_size=group, residual=group, capacity=64, batch=batch)
    c = quant.quantize_kv(k, v, bits=bits, group=group, residual=group)
    return (tkv.SharedPrefix(P, L), np.concatenate([quant.dequantize_k(c), c.k_resid.astype(np.float64)], axis=1),
            np.concatenate([quant.dequantize_v(c), c.v_resid.astype(np.float64)], axis=1))


@pytest.mark.parametrize("bits,group", SETTINGS)
@pytest.mark.parametrize("batch", BATCHES)
def test_keys(batch, bits, group):
    """Channels in pairs, the second 1.5 times the first, queries (12, -8) times a sign: q.k is 0 but for the scalers' own
    rounding to fp16 (and, seldom, a code's).  Logits are exact but for their scaling (1.5 2^-23 of at most 100): a weight is rounded to fp16 (2^-11), the output too.
    K-hat rounded to fp16 (half a step 2^-5 at 64 and above, times 12 in 128 channels) would be a logit off by about 0.2."""
    print(f"case keys {bits} bit/{group} batch {batch}", flush=True)
    r = np.random.default_rng(bits * group + batch)
    n = 2 * 64 + group
    k = np.zeros((2, n, 128))
    k[:, :, ::2] = r.integers(-400, 401, (2, n, 64)) / 4.0
    k[:, :, 1::2] = 1.5 * k[:, :, ::2]
    v = r.standard_normal((2, n, 128)).astype(np.float16)
    q = np.zeros((batch, 16, 128))
    q[:, :, ::2] = 12 * r.choice([-1, 1], (batch, 16, 64))
    q[:, :, 1::2] = q[:, :, ::2] / -1.5
    plan, kk, vv = _layers(k.astype(np.float16), v, bits, group, batch)
    out = plan.attn_decode(torch.from_numpy(q.astype(np.float16)).cuda(), SM).double().cpu().numpy()
    for b in range(batch):
        ref, size = (attention.decode_attention(q[b], kk, x, SM) for x in (vv, np.abs(vv)))
        assert np.abs(np.einsum("hc,htc->ht", q[b, ::8], kk)).max() * SM < 100
        # (a weight's rounding moves numerator and sum: |v - out| of it; 2^-15: the exponent's and the sums' float32 errors)
        bound = 2.0 ** -11 * np.abs(ref) + (2.0 ** -11 + 2.0 ** -15) * (size + np.abs(ref)) + 2.0 ** -25
        assert (np.abs(out[b] - ref) <= bound).all(), float((np.abs(out[b] - ref) / bound).max())


@pytest.mark.parametrize("bits,group", SETTINGS)
@pytest.mark.parametrize("batch", BATCHES)
def test_values(batch, bits, group):
    """Rows in threes, u, -0.375 u and -0.625 u, and queries of zero: all weights are 2^7, the output is the mean, small beside the
    values, and exact but for its rounding to fp16 (2^-11) and the division (2^-22).  V-hat rounded to fp16 (half a step 2^-5 at 64
    and above) would move the mean by about 1e-3."""
    print(f"case values {bits} bit/{group} batch {batch}", flush=True)
    r = np.random.default_rng(bits * group + batch)
    n = 96 + group if group == 32 else 192 + group
    u = r.integers(-512, 513, (2, n // 3 + 1, 128)) / 4.0
    v = (u[:, :, None] * np.array([1, -0.375, -0.625])[None, None, :, None]).reshape(2, -1, 128)[:, :n].astype(np.float16)
    k = r.standard_normal((2, n, 128)).astype(np.float16)
    plan, kk, vv = _layers(k, v, bits, group, batch)
    out = plan.attn_decode(torch.zeros(batch, 16, 128, dtype=torch.float16, device="cuda"), SM).double().cpu().numpy()
    ref = np.repeat(vv.mean(axis=1), 8, axis=0)
    bound = (2.0 ** -11 + 2.0 ** -21) * np.abs(ref) + 2.0 ** -25
    assert (np.abs(out - ref) <= bound).all(), float((np.abs(out - ref) / bound).max())
