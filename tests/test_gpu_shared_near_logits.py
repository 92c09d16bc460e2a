"""tkv_quant_attn_decode_shared with logits of the documented size, up to 2^26, that lie near each other and rise with the token, so that
some are above a wave's reference by about as much as a weight may grow: weights stay finite.

A step of float32 is a logit's 1 and more there, and what is asked for is what that leaves: a mean of the dequantized values (of magnitude M
at most) with some weights, rounded once each (half a step u of fp16, relative), rounded itself: at most (1 + u)^2 M."""
import numpy as np
import pytest
import torch

import paper_2505_19586_amd as tkv
from oracle import quant

from gpu_util import to_new

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits,group", [(1, 32), (1, 64), (2, 32), (2, 64), (4, 32), (4, 64)])
@pytest.mark.parametrize("batch", [1, 9])  # of eight query heads per KV head: 8 and 72 rows
@pytest.mark.parametrize("n", [400, 20000])
def test_near_logits_far_out(n, batch, bits, group):
    print(f"case {n} tokens batch {batch} {bits} bit/{group}, near logits to 2^26", flush=True)
    r = np.random.default_rng(bits * group + batch)
    v = r.standard_normal((2, n, 128)).astype(np.float16)
    own = tkv.QuantLayer(n_q_heads=16, n_kv_heads=2, bits=bits, group_size=group, capacity=64, batch=batch)
    most = None
    for top in (23, 24, 25, 26):
        for sign in (1.0, -1.0):
            k = np.zeros((2, n, 128), np.float16)
            k[..., 3] = sign * 2.0 ** (top - 13)
            # one of two neighbours in every group: quantized without a rounding
            level = np.arange(n) // group * 24 // (n // group + 1)
            k[..., 40] = max(1.0, 2.0 ** (top - 24)) * (level + r.integers(0, 2, (2, n)))
            q = np.zeros((batch, 16, 128), np.float16)
            q[..., 3] = 4.0 * r.integers(1024, 2048, (batch, 16))
            q[..., 40] = 1
            shared = tkv.QuantLayer(n_q_heads=16, n_kv_heads=2, bits=bits, group_size=group, capacity=-(-n // 64) * 64 + 64)
            shared.append(to_new(k), to_new(v))
            out = tkv.SharedPrefix(shared, own).attn_decode(torch.from_numpy(q).cuda(), 1.0).double().cpu().numpy()
            if most is None:
                c = quant.quantize_kv(k, v, bits=bits, group=group, residual=128)
                most = (1 + 2.0 ** -11) ** 2 * max(np.abs(quant.dequantize_v(c)).max(), np.abs(c.v_resid.astype(np.float64)).max())
            assert (np.abs(out) <= most).all(), (top, sign)
