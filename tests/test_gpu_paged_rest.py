"""tkv_paged_attn: rows of outputs that nobody attends for."""
import pytest
import torch

import paper_2505_19586_amd as tkv

pytestmark = pytest.mark.gpu
SM = 128 ** -0.5


@pytest.mark.parametrize("batch", [2, 700])
def test_rows_beyond_the_most_that_a_sequence_may_have_are_of_none(batch):
    """New outputs hold zeros and -inf there, given ones what they held; more sequences than workgroups."""
    print(f"case rows beyond max_q_len, {batch} sequences", flush=True)
    cache = tkv.PagedCache(n_q_heads=4, n_kv_heads=2, n_pages=1)
    cache.v_pages[0, :, :5] = 3
    q = torch.randn(6 * batch, 4, 128, device="cuda").half()
    starts = 6 * torch.arange(batch + 1, device="cuda", dtype=torch.int32)
    table, lens = torch.zeros(batch, 1, device="cuda", dtype=torch.int32), torch.full((batch,), 5, device="cuda", dtype=torch.int32)

    def rows(x):
        x = x.view(batch, 6, *x.shape[1:])
        return x[:, :2], x[:, 2:]

    junk = [torch.full(s, float("nan"), dtype=d, device="cuda") for s, d in ((q.shape, torch.float16), ((6 * batch, 4), torch.float32))]
    del junk                                                              # (what a new tensor's memory may hold)
    out, lse = cache.attend(q, SM, table, lens, q_starts=starts, max_q_len=2, lse=True)
    torch.cuda.synchronize()
    (have, rest), (lse_have, lse_rest) = rows(out), rows(lse)
    assert (have == 3).all() and not rest.any() and lse_have.isfinite().all() and torch.isneginf(lse_rest).all()
    out, lse = torch.full_like(q, 7.0), torch.full((6 * batch, 4), 5.0, device="cuda")
    cache.attend(q, SM, table, lens, q_starts=starts, max_q_len=2, out=out, lse=lse)
    torch.cuda.synchronize()
    (have, rest), (_, lse_rest) = rows(out), rows(lse)
    assert (have == 3).all() and (rest == 7).all() and (lse_rest == 5).all()


@pytest.mark.parametrize("most", [7, 2**31 - 1, 2**31, 2**32 + 1, 2**63 - 1, 2**64 + 2])
def test_any_bound_on_queries(most):
    """Numbers beyond 32 bits too."""
    print(f"case max_q_len {most}", flush=True)
    cache = tkv.PagedCache(n_q_heads=4, n_kv_heads=2, n_pages=1)
    for x in (cache.k_pages, cache.v_pages):
        x.normal_(generator=torch.Generator(device="cuda").manual_seed(0))
    q = torch.randn(9, 4, 128, device="cuda").half()
    starts = torch.tensor([0, 2, 9], device="cuda", dtype=torch.int32)
    table, lens = torch.zeros(2, 1, device="cuda", dtype=torch.int32), torch.tensor([5, 60], device="cuda", dtype=torch.int32)
    got = cache.attend(q, SM, table, lens, q_starts=starts, max_q_len=most)
    want = cache.attend(q, SM, table, lens, q_starts=starts, max_q_len=7)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and want.any(2).all()


@pytest.mark.parametrize("low", [-2**31, -2**31 + 1, -2**31 + 40, -1])
def test_starts_far_below_zero_reach_nothing(low):
    """Invalid, but nothing out of bounds is touched: where one sequence would end below zero it has no rows, however far below."""
    print(f"case starts with {low}", flush=True)
    cache = tkv.PagedCache(n_q_heads=4, n_kv_heads=2, n_pages=1)
    cache.v_pages[0, :, :5] = 3
    q = torch.randn(5, 4, 128, device="cuda").half()
    table, lens = torch.zeros(5, 1, device="cuda", dtype=torch.int32), torch.full((5,), 5, device="cuda", dtype=torch.int32)
    whole, whole_lse = torch.full((64, 4, 128), 7.0, device="cuda").half(), torch.full((64, 4), 5.0, device="cuda")
    for at in range(1, 6):                                # (the sequence in front of it would end there)
        starts = torch.arange(6, device="cuda", dtype=torch.int32)
        starts[at] = low
        cache.attend(q, SM, table, lens, q_starts=starts, max_q_len=3, out=whole[:5], lse=whole_lse[:5])
        cache.attend(q, SM, table, lens, q_starts=starts, max_q_len=3)
        torch.cuda.synchronize()
        assert (whole[5:] == 7).all() and (whole_lse[5:] == 5).all(), at
        rows = [b for b in range(5) if b != at - 1 and b != at]
        assert (whole[rows] == 3).all(), at
