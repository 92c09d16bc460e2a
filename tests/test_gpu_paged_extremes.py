"""tkv_paged_attn with logits of the documented size, up to 2^26, that lie near each other: weights that matter, references that move.

Two channels of q and k are not 0: a large product that all keys of a sequence share, and a small one, a whole number of float32's steps at
the large one's size.  So every logit is exact in float32, and the weights follow from their differences: tolerances are those of
ordinary logits (half a step of the type for a weight and for the output; what float32 adds, a difference of up to 64 times the scale's
2^-24 and the exponents' own roundings, is within the tenth of a half step).  The logarithm of the sum is near 2^26: 2^-20 of it (a handful of
float32 roundings)."""
import numpy as np
import pytest
import torch

import paper_2505_19586_amd as tkv
from oracle import paged
from oracle.prompt import prompt_attention

pytestmark = pytest.mark.gpu
HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
BOTH = pytest.mark.parametrize("bits", [16, 4])


def _f64(x):
    return x.double().cpu().numpy()


def _compare(out, lse, q, k, v, dtype, sm):
    ref, ref_lse = prompt_attention(q, k, v, sm)
    size, _ = prompt_attention(q, k, np.abs(v), sm)
    u = HALF_STEP[dtype]
    tiny = 2.0 ** -25 if dtype == torch.float16 else 0.0
    assert (np.abs(_f64(out) - ref) <= u * np.abs(ref) + 1.1 * u * size + tiny).all()
    assert (np.abs(_f64(lse) / ref_lse - 1) <= 2.0 ** -20).all()


def near_logits(n, top, sign, rng):
    """(the shared product's factor for a query channel of 4096 to 8160, n small products): logits from 2^(top - 1) to 2^top, which rise
    with the key, now and then by several steps."""
    grid = np.array([0, 1, 2, 3, 4, 6, 8, 12, 16])        # (one bit of mantissa behind the first: exact in 4 bits too)
    step = max(1.0, 2.0 ** (top - 24))
    at = np.clip(9 * np.arange(n) // n - rng.integers(0, 3, n), 0, 8)
    return sign * 2.0 ** (top - 13), step * grid[at]


@BOTH
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("nq,n", [(1, 320), (1, 9000), (5, 3000)])
def test_near_logits_far_out(nq, n, dtype, bits):
    print(f"case {nq} over {n} {dtype} {bits} bits, logits to 2^26", flush=True)
    rng = np.random.default_rng(n)
    hq, hkv, page = 8, 2, 64
    cases = [(top, sign) for top in (20, 23, 24, 25, 26) for sign in (1.0, -1.0)]
    each = -(-n // page)
    cache = tkv.PagedCache(n_q_heads=hq, n_kv_heads=hkv, page_size=page, bits=bits, dtype=dtype, n_pages=each * len(cases))
    table = torch.arange(each * len(cases), dtype=torch.int32).view(len(cases), each)
    g = torch.Generator(device="cuda").manual_seed(n)
    rows = []
    for b, (top, sign) in enumerate(cases):
        k = np.zeros((n, hkv, 128))
        for h in range(hkv):
            k[:, h, 3], k[:, h, 40] = near_logits(n, top, sign, rng)
        k = torch.from_numpy(k).cuda().to(dtype)
        v = torch.randn(n, hkv, 128, generator=g, device="cuda").to(dtype)
        slots = torch.from_numpy(paged.sequence_slots(table[b].numpy(), n, page).astype(np.int32)).cuda()
        cache.append(None, k, v, slots)
        got = cache.gather(slots)
        assert torch.equal(got[0], k)
        rows.append((_f64(k), _f64(got[1])))
    q = torch.zeros(nq * len(cases), hq, 128, device="cuda", dtype=dtype)
    # (eight bits: exact in both types)
    q[..., 3] = torch.from_numpy(32.0 * rng.integers(128, 256, (nq * len(cases), hq))).to(dtype).cuda()
    q[..., 40] = 1
    lens = torch.full((len(cases),), n, device="cuda", dtype=torch.int32)
    starts = nq * torch.arange(len(cases) + 1, device="cuda", dtype=torch.int32)
    out, lse = cache.attend(q, 1.0, table.cuda(), lens, q_starts=starts, max_q_len=nq, lse=True)
    torch.cuda.synchronize()
    for b, (k, v) in enumerate(rows):
        i, j = nq * b, nq * (b + 1)
        _compare(out[i:j], lse[i:j], _f64(q[i:j]), k, v, dtype, 1.0)


@pytest.mark.parametrize("far", [31, 32, 100, 159])
def test_a_later_key_just_above_a_far_reference(far):
    """Logits of 1.2e7 whose exponents, of 2, differ by 8 after float32's rounding and by more before: inside fp16 all the same.  Enough
    sequences, over the same pages, that a wave takes several tiles of one."""
    sm, batch = 128 ** -0.5, 1200
    k = torch.zeros(far + 1, 1, 128, device="cuda").half()
    k[:, 0, 0] = 2234
    k[far, 0, 1] = 64
    v = torch.randn(far + 1, 1, 128, generator=torch.Generator(device="cuda").manual_seed(0), device="cuda").half()
    q = torch.zeros(batch, 4, 128, device="cuda").half()
    q[..., 0], q[..., 1] = 60000, 1                      # (q.k: 134040000 and 134040064, both exact in float32)
    cache = tkv.PagedCache(n_q_heads=4, n_kv_heads=1, n_pages=3)
    cache.append(None, k, v, torch.arange(far + 1, device="cuda", dtype=torch.int32))
    table = torch.tensor([[0, 1, 2]], device="cuda", dtype=torch.int32).repeat(batch, 1)
    out, lse = cache.attend(q, sm, table, torch.full((batch,), far + 1, device="cuda", dtype=torch.int32), lse=True)
    torch.cuda.synchronize()
    for b in range(0, batch, 100):
        _compare(out[b:b + 1], lse[b:b + 1], _f64(q[b:b + 1]), _f64(k), _f64(v), torch.float16, sm)
    assert (out == out[0]).all()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("batch,nq,n", [(1, 1, 5), (1, 1, 9000), (300, 1, 400), (40, 7, 3), (2, 5, 3000)])
def test_logits_of_minus_infinity(batch, nq, n, dtype):
    """Rows whose every key has a logit of -infinity: 0 / 0, not the zeros of rows without keys; with one finite logit among them, its
    key's value."""
    print(f"case {batch} times {nq} over {n} {dtype}, logits of -inf", flush=True)
    page = 64
    each = -(-n // page)
    cache = tkv.PagedCache(n_q_heads=8, n_kv_heads=2, page_size=page, dtype=dtype, n_pages=each)
    k = torch.ones(n, 2, 128, device="cuda", dtype=dtype)
    k[:, :, 7] = -float("inf")
    k[n // 2, 1, 7] = 2                                   # (the second head's)
    v = torch.randn(n, 2, 128, generator=torch.Generator(device="cuda").manual_seed(n), device="cuda").to(dtype)
    cache.append(None, k, v, torch.arange(n, device="cuda", dtype=torch.int32))
    q = torch.ones(batch * nq, 8, 128, device="cuda", dtype=dtype)
    table = torch.arange(each, device="cuda", dtype=torch.int32).repeat(batch, 1)
    lens = torch.full((batch,), n, device="cuda", dtype=torch.int32)
    starts = nq * torch.arange(batch + 1, device="cuda", dtype=torch.int32)
    out, lse = cache.attend(q, 128 ** -0.5, table, lens, q_starts=starts, max_q_len=nq, lse=True)
    torch.cuda.synchronize()
    out, lse = out.view(batch, nq, 2, 4, 128), lse.view(batch, nq, 2, 4)
    last = torch.arange(nq, device="cuda") + n - nq       # last key that a query sees
    seen, one = last >= 0, last >= n // 2
    assert not out[:, ~seen].any() and torch.isneginf(lse[:, ~seen]).all()
    assert out[:, seen, 0].isnan().all() and torch.isneginf(lse[:, seen, 0]).all()
    assert out[:, seen & ~one, 1].isnan().all()
    assert (out[:, one, 1] == v[n // 2, 1]).all() and lse[:, one, 1].isfinite().all()
