"""Where every value row holds one number, tkv_quant_attn_decode_shared returns that number: it divides by the sum of the weights as
they multiply the values, rounded ones, of quantized tokens and of those still in the ring alike.

c = 2 - 2^-10, the keys two rows in turn, so that nearly all weights of a query are the same number and rounded the same way: divided by
the sum of the unrounded weights, the output would be off by that rounding, up to 2^-11 of it, where c's neighbours are half as far
away.  With the rounded sum only float32's errors remain: products of 16-bit numbers are exact; up to 1024 keys between two
roundings of a part's sums, (1024 / 32) (32 + 1) 2^-24 < 2^-13 of numerator and sum together, half of the half step that would show."""
import pytest
import torch

import paper_2505_19586_amd as tkv

pytestmark = pytest.mark.gpu
SM = 128 ** -0.5
C = 2 - 2.0 ** -10


def _two_keys(n, heads, gen, every=37):
    """Rows of one key, every 37th of another."""
    two = torch.randn(2, heads, 128, generator=gen, device="cuda").half()
    return two[(torch.arange(n, device="cuda") % every == 0).long()].contiguous()


@pytest.mark.parametrize("bits,group", [(1, 32), (1, 64), (2, 32), (2, 64), (4, 32), (4, 64)])
@pytest.mark.parametrize("n_prefix,lens", [(0, [100, 1, 37]), (900, [150, 0, 64]), (100, [700, 20, 64])])
def test_shared(n_prefix, lens, bits, group):
    """Tokens still in the ring, quantized ones and both together (values all alike are quantized to themselves)."""
    print(f"case shared {n_prefix} + {lens} {bits} bit/{group}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(n_prefix + bits)

    def layer(lens):
        L = tkv.QuantLayer(n_q_heads=16, n_kv_heads=4, bits=bits, group_size=group, capacity=1024, batch=len(lens))
        if max(lens):
            k = torch.stack([_two_keys(max(lens), 4, gen) for _ in lens])
            L.append(k, torch.full_like(k, C), n_valid=lens)
        return L

    q = torch.randn(len(lens), 16, 128, generator=gen, device="cuda").half()
    P, L = layer([n_prefix]), layer(lens)
    out = tkv.SharedPrefix(P, L).attn_decode(q, SM)
    want = torch.full_like(out, C)
    want[[b for b, n in enumerate(lens) if n + n_prefix == 0]] = 0
    assert torch.equal(out, want), float((out.float() - want.float()).abs().max())
