"""tkv_prompt_attn with logits near the ends of float32's range (bfloat16 rows reach them): the largest weight is 1 wherever the logits lie.

One channel of q and k is not 0, so that a logit is one product, and all of a row are the same number L: weights are exactly 1/n, the output is the
mean (half a step 2^-8 of it, 2^-20 of the values for the sums), the logarithm of the sum L + log n, which is L in float32 (to 2^-20)."""
import pytest
import torch

import paper_2505_19586_amd as tkv

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("logit", [-2.0 ** 125, -2.0 ** 110, -2.0 ** 100, 2.0 ** 100, 2.0 ** 125])
@pytest.mark.parametrize("nq,nk", [(1, 1), (1, 70), (1, 9000), (100, 300), (64, 9000)])
def test_one_logit_far_out(nq, nk, logit):
    """Both kernels, keys whole and in pieces."""
    print(f"case {nq} over {nk}, logits {logit:g}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(nk)
    q, k = (torch.zeros(n, h, 128, dtype=torch.bfloat16, device="cuda") for n, h in ((nq, 8), (nk, 2)))
    q[..., 5], k[..., 5] = 2.0 ** 62, logit / 2.0 ** 62
    v = torch.randn(nk, 2, 128, generator=g, device="cuda").bfloat16()
    plan = tkv.PromptAttention(n_q_heads=8, n_kv_heads=2, dtype=torch.bfloat16, causal=False)
    out, lse = plan.attend(q, k, v, 1.0, [nq], [nk], lse=True)
    ref = v.double().mean(0).repeat_interleave(4, 0)
    size = v.double().abs().mean(0).repeat_interleave(4, 0)
    assert ((out.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -20 * size).all()
    assert ((lse.double() / logit - 1).abs() <= 2.0 ** -20).all()
