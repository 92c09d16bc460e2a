"""tkv_prompt_attn with logits far out: rows that have keys are told from rows that have none wherever their logits lie, and logits up to
2^26 are weighed whatever they are.

One channel of q and k is not 0, so that a logit is one product.  The same number L, a power of two, for all of a row (bfloat16 reaches
the ends of float32's range): weights are exactly 1/n, the output is the mean (half a step 2^-8 of it, 2^-20 of the values for the sums),
the logarithm of the sum L + log n, which is L in float32 (to 2^-20)."""
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


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("nq,nk", [(1, 70), (1, 9000), (100, 300), (64, 9000)])
def test_any_logits_up_to_the_documented_size(nq, nk, dtype):
    """Products are exact in float32; as far out as this, logits that differ give weights of 1 and 0, equal ones equal weights: the output is
    off by a weight's rounding and its own (half a step each)."""
    print(f"case {nq} over {nk} {dtype}, logits up to 2^26", flush=True)
    g = torch.Generator(device="cuda").manual_seed(nk)

    def rows(n, h):
        x = torch.zeros(n, h, 128, dtype=dtype, device="cuda")
        size = 2.0 ** (12 + torch.rand(n, h, generator=g, device="cuda"))
        x[..., 5] = (size * torch.where(torch.rand(n, h, generator=g, device="cuda") < 0.5, -1.0, 1.0)).to(dtype)
        return x

    q, k, v = rows(nq, 8), rows(nk, 2), torch.randn(nk, 2, 128, generator=g, device="cuda").to(dtype)
    out, lse = tkv.PromptAttention(n_q_heads=8, n_kv_heads=2, dtype=dtype, causal=False).attend(q, k, v, 1.0, [nq], [nk], lse=True)
    u = 2.0 ** -11 if dtype == torch.float16 else 2.0 ** -8
    for h in range(8):
        s = q[:, h, 5:6].double() * k[None, :, h // 4, 5].double()
        w = torch.softmax(s, 1)
        ref, size = w @ v[:, h // 4].double(), w @ v[:, h // 4].double().abs()
        assert ((out[:, h].double() - ref).abs() <= u * ref.abs() + 1.1 * u * size + 2.0 ** -25).all()
        assert ((lse[:, h].double() / torch.logsumexp(s, 1) - 1).abs() <= 2.0 ** -20).all()
