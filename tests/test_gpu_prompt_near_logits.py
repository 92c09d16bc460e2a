"""tkv_prompt_attn with logits of the documented size, up to 2^26, that lie near each other, where a key's logit is above a reference by
about as much as a weight may grow: weights stay finite.

Two channels of q and k are not 0: a large product that all keys share, and a small one, a whole number of float32's steps at the large
one's size, so that every logit is exact in float32.  Beyond 2^23 a step of float32 is a logit's 1 and more, and what is asked for is
what that leaves: a mean of the values with some weights, each rounded once (half a step u of the type, relative), rounded itself: at most
(1 + u)^2 times the largest magnitude.  The logarithm of the sum: within 2^-20 (a few float32 roundings of the logit's size)."""
import numpy as np
import pytest
import torch

import paper_2505_19586_amd as tkv

pytestmark = pytest.mark.gpu
HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("nq,nk", [(1, 320), (1, 9000), (6, 40000), (100, 320), (64, 9000), (300, 700)])
def test_near_logits_far_out(nq, nk, dtype):
    """Few rows and many, keys whole and in pieces; the rows of a sequence have different logits."""
    print(f"case {nq} over {nk} {dtype}, near logits to 2^26", flush=True)
    rng = np.random.default_rng(nk)
    hq, hkv, u = 8, 2, HALF_STEP[dtype]
    grid = np.array([0, 1, 2, 3, 4, 6, 8, 12, 16])
    g = torch.Generator(device="cuda").manual_seed(nk)
    plan = tkv.PromptAttention(n_q_heads=hq, n_kv_heads=hkv, dtype=dtype, causal=False)
    q = torch.zeros(nq, hq, 128, device="cuda", dtype=dtype)
    q[..., 3] = torch.from_numpy(32.0 * rng.integers(128, 256, (nq, hq))).to(dtype).cuda()   # (eight bits: exact in both types)
    q[..., 40] = 1
    v = torch.randn(nk, hkv, 128, generator=g, device="cuda").to(dtype)
    most = (1 + u) ** 2 * v.double().abs().amax(0).repeat_interleave(hq // hkv, 0)
    for top in (20, 23, 24, 25, 26):
        for sign in (1.0, -1.0):
            k = np.zeros((nk, hkv, 128))
            k[..., 3] = sign * 2.0 ** (top - 13)
            at = np.clip(9 * np.arange(nk)[:, None] // nk - rng.integers(0, 3, (nk, hkv)), 0, 8)      # (logits rise with the key)
            k[..., 40] = max(1.0, 2.0 ** (top - 24)) * grid[at]
            k = torch.from_numpy(k).cuda().to(dtype)
            out, lse = plan.attend(q, k, v, 1.0, [nq], [nk], lse=True)
            torch.cuda.synchronize()
            assert (out.double().abs() <= most).all(), (top, sign)
            s = torch.stack([q[:, h].double() @ k[:, h // 4].double().T for h in range(hq)])
            assert ((lse.double() / torch.logsumexp(s, 2).T - 1).abs() <= 2.0 ** -20).all(), (top, sign)


@pytest.mark.parametrize("far", [31, 32, 100, 159, 300])
@pytest.mark.parametrize("nq", [1, 40])
def test_a_later_key_just_above_a_far_reference(nq, far):
    """Logits of 1.2e7 whose exponents, of 2, differ by 8 after float32's rounding and by more before: inside fp16 all the same.  Enough
    sequences, over the same keys, that a wave takes several tiles of one."""
    print(f"case {nq} with key {far} above the others", flush=True)
    sm, batch, u = 128 ** -0.5, 50, 2.0 ** -11
    k = torch.zeros(far + 1, 2, 128, device="cuda").half()
    k[:, :, 0] = 2234
    k[far, :, 1] = 64
    v = torch.randn(far + 1, 2, 128, generator=torch.Generator(device="cuda").manual_seed(0), device="cuda").half()
    q = torch.zeros(batch * nq, 8, 128, device="cuda").half()
    q[..., 0], q[..., 1] = 60000, 1                      # (q.k: 134040000 and 134040064, both exact in float32)
    plan = tkv.PromptAttention(n_q_heads=8, n_kv_heads=2, causal=False, batch=batch)
    out = plan.attend(q, k, v, sm, [nq] * batch, [far + 1] * batch, k_starts=[0] * batch)
    torch.cuda.synchronize()
    assert (out.double().abs() <= (1 + u) ** 2 * v.double().abs().amax(0).repeat_interleave(4, 0)).all()
