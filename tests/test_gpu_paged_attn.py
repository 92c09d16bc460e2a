"""tkv_paged_attn against float64: lengths from none to many tiles, page sizes, head groups, types, drafts and chunks, what lies behind
a sequence's tokens, pages that are shared or outside, streams and replayed graphs.

Tolerance: with u = half a step of the type (fp16 2^-11, bf16 2^-8), a weight is rounded once (u, relative), the output once
(u, relative), the sums and logits are float32 (products of 16-bit numbers are exact there, and 4-bit codes stand for such): |o - ref| <=
u |ref| + 1.1 u sum_j w_j |v_j|, w the exact weights.  The logarithm of the sum: 1e-5 absolute (float32 logits of magnitude up to 32:
128 terms, 2^-24 each)."""
import numpy as np
import pytest
import torch

import paper_2505_19586_amd as tkv
from oracle import paged
from oracle.prompt import prompt_attention

pytestmark = pytest.mark.gpu
SM = 128 ** -0.5
HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def _f64(x):
    return x.double().cpu().numpy()


def _compare(out, lse, q, k, v, dtype, sm=SM):
    ref, ref_lse = prompt_attention(q, k, v, sm)
    size, _ = prompt_attention(q, k, np.abs(v), sm)
    u = HALF_STEP[dtype]
    tiny = 2.0 ** -25 if dtype == torch.float16 else 0.0
    err = np.abs(_f64(out) - ref)
    assert (err <= u * np.abs(ref) + 1.1 * u * size + tiny).all(), float((err / (u * size + 1e-30)).max())
    lse = _f64(lse)
    assert np.array_equal(np.isneginf(lse), np.isneginf(ref_lse))
    seen = np.isfinite(ref_lse)
    assert np.abs(lse[seen] - ref_lse[seen]).max(initial=0.0) <= 1e-5


def _filled(k_lens, hkv, page, bits, dtype, seed=0, spare=3):
    """A cache whose sequences' tokens lie in pages in any order, NaN in every slot behind them: cache, table, k, v (float64, by sequence)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    used = [-(-n // page) for n in k_lens]
    n_pages = sum(used) + spare
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).tolist()
    each = max(max(used), 1)
    table = torch.full((len(k_lens), each), 2**31 - 1, dtype=torch.int32)    # (never looked at behind the last page)
    nan = float("nan")
    if bits == 16:
        pages = [torch.full((n_pages, hkv, page, 128), nan, device="cuda").to(dtype) for _ in range(2)]
    else:
        pages = [torch.full((n_pages, hkv, 68 * page), 255, device="cuda", dtype=torch.uint8) for _ in range(2)]
    cache = tkv.PagedCache(n_q_heads=hkv, n_kv_heads=hkv, page_size=page, bits=bits, dtype=dtype, k_pages=pages[0], v_pages=pages[1])
    rows, at = [], 0
    for b, n in enumerate(k_lens):
        table[b, :used[b]] = torch.tensor(order[at:at + used[b]], dtype=torch.int32)
        at += used[b]
        k, v = ((torch.randn(n, hkv, 128, generator=g, device="cuda") * gain).to(dtype) for gain in (1.0, 1.0))
        slots = torch.from_numpy(paged.sequence_slots(table[b].numpy(), n, page).astype(np.int32)).cuda()
        cache.append(None, k, v, slots)
        if bits == 4:
            k, v = cache.gather(slots)
        rows.append((_f64(k), _f64(v)))
    return pages, table.cuda(), rows


def _run(q_lens, k_lens, hq, hkv, page=64, bits=16, dtype=torch.float16, seed=0, starts=True, most=None):
    pages, table, rows = _filled(k_lens, hkv, page, bits, dtype, seed)
    cache = tkv.PagedCache(n_q_heads=hq, n_kv_heads=hkv, page_size=page, bits=bits, dtype=dtype, k_pages=pages[0], v_pages=pages[1])
    g = torch.Generator(device="cuda").manual_seed(seed + 100)
    q = torch.randn(sum(q_lens), hq, 128, generator=g, device="cuda").to(dtype)
    lens = torch.tensor(k_lens, device="cuda", dtype=torch.int32)
    at = torch.tensor([0, *np.cumsum(q_lens)], device="cuda", dtype=torch.int32) if starts else None
    out, lse = cache.attend(q, SM, table, lens, q_starts=at, max_q_len=most or max(max(q_lens), 1), lse=True)
    torch.cuda.synchronize()
    x = _f64(q)
    q0 = 0
    for nq, (k, v) in zip(q_lens, rows):
        _compare(out[q0:q0 + nq], lse[q0:q0 + nq], x[q0:q0 + nq], k, v, dtype)
        q0 += nq
    again, lse2 = cache.attend(q, SM, table, lens, q_starts=at, max_q_len=most or max(max(q_lens), 1), lse=True)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    return cache, q, table, lens, out


BOTH = pytest.mark.parametrize("bits", [16, 4])


@BOTH
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 500, 1030])
def test_single_tokens(n, dtype, bits):
    print(f"case single token over {n} {dtype} {bits} bits", flush=True)
    _run([1], [n], 8, 2, 16 if n % 2 else 64, bits, dtype, seed=n, starts=False)


@BOTH
@pytest.mark.parametrize("page", [16, 32, 64, 128, 1024])
def test_page_sizes_and_lengths_of_a_batch(page, bits):
    print(f"case page {page} {bits} bits", flush=True)
    _run([1] * 9, [700, 1, 0, 33, 1025, 64, 300, 128, 15], 8, 2, page, bits, seed=page, starts=False)


@BOTH
@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (5, 5), (14, 2), (16, 1), (17, 1), (33, 1), (64, 1), (80, 1), (32, 4)])
def test_head_groups(hq, hkv, bits):
    print(f"case heads {hq}/{hkv} {bits} bits", flush=True)
    _run([1, 1], [150, 333], hq, hkv, 32, bits, seed=hq, starts=False)
    _run([2, 5], [90, 170], hq, hkv, 32, bits, seed=hq)


@BOTH
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_drafts_chunks_and_empty_sequences(dtype, bits):
    print(f"case drafts {dtype} {bits} bits", flush=True)
    _run([1, 0, 5, 3, 64, 1, 8, 2], [1, 70, 130, 300, 64, 515, 0, 1], 8, 2, 16, bits, dtype, seed=3)


@BOTH
@pytest.mark.parametrize("nq,nk", [(100, 37), (100, 100), (150, 700), (1, 3000), (7, 2111)])
def test_chunks_longer_than_a_tile_of_rows(nq, nk, bits):
    print(f"case chunk {nq} over {nk} {bits} bits", flush=True)
    _run([nq], [nk], 8, 2, 64, bits, seed=nk)


@BOTH
def test_many_sequences(bits):
    """More than a wave has lanes, and more than a workgroup has threads."""
    print(f"case many sequences {bits} bits", flush=True)
    lens = [(37 * b) % 90 for b in range(130)]
    _run([1] * 130, lens, 4, 1, 16, bits, seed=1, starts=False)
    _run([b % 3 for b in range(300)], [(b * 7) % 40 for b in range(300)], 2, 1, 16, bits, seed=2)


@BOTH
def test_one_long_sequence_among_short_ones(bits):
    print(f"case ragged {bits} bits", flush=True)
    _run([1] * 20, [20011] + [5 + b for b in range(19)], 8, 2, 64, bits, seed=4, starts=False)


@BOTH
def test_long_single_sequence(bits):
    print(f"case long {bits} bits", flush=True)
    _run([1], [33333], 4, 1, 64, bits, seed=5, starts=False)
    _run([3], [9000], 8, 2, 64, bits, torch.bfloat16, seed=6)


def test_a_bound_on_queries_that_is_not_reached_or_too_small():
    """max_q_len is what the host knows: any bound does; more queries than it says count as that many."""
    for most in (40, 41, 100, 1 << 30):
        _run([3, 1, 40], [50, 77, 130], 8, 2, 32, 16, seed=7, most=most)
    cache, q, table, lens, _ = _run([3, 1, 40], [50, 77, 130], 8, 2, 32, 16, seed=7)
    got = cache.attend(q, SM, table, lens, q_starts=torch.tensor([0, 3, 4, 44], device="cuda", dtype=torch.int32), max_q_len=2)
    want = cache.attend(torch.cat((q[:2], q[3:6])), SM, table, lens, q_starts=torch.tensor([0, 2, 3, 5], device="cuda", dtype=torch.int32), max_q_len=2)
    torch.cuda.synchronize()
    assert torch.equal(torch.cat((got[:2], got[3:6])), want)


def test_starts_that_do_not_ascend_end():
    """Invalid, but nothing out of bounds is touched and every wave ends: rows of sequences that are sound come out."""
    cache, q, table, lens, want = _run([1] * 5, [50, 77, 130, 9, 64], 8, 2, 32, 16, seed=7)
    for starts in ([0, 1, 2, 1, 4, 5], [-7, 1, 2, 3, 4, 5], [0, 1, 2, 3, 4, 1 << 30], [5, 4, 3, 2, 1, 0]):
        got = cache.attend(q, SM, table, lens, q_starts=torch.tensor(starts, device="cuda", dtype=torch.int32), max_q_len=3)
        torch.cuda.synchronize()
        if starts[1:4] == [1, 2, 3]:
            assert torch.equal(got[1], want[1])


def test_rows_of_no_sequence_are_left():
    cache, q, table, lens, want = _run([2, 3], [40, 50], 4, 2, 16, 16, seed=8)
    wide = torch.randn(9, 4, 128, device="cuda").half()
    wide[2:7] = q
    starts = torch.tensor([2, 4, 7], device="cuda", dtype=torch.int32)
    out, lse = torch.full_like(wide, 7.0), torch.full((9, 4), 5.0, device="cuda")
    got = cache.attend(wide, SM, table, lens, q_starts=starts, max_q_len=3, out=out, lse=lse)
    torch.cuda.synchronize()
    assert got[0] is out and torch.equal(out[2:7], want)
    assert (out[:2] == 7).all() and (out[7:] == 7).all() and (lse[:2] == 5).all() and (lse[7:] == 5).all() and lse[2:7].isfinite().all()
    for given in (dict(), dict(lse=True), dict(lse=torch.full((9, 4), 5.0, device="cuda")), dict(out=torch.full_like(wide, 7.0), lse=True)):
        junk = torch.full((1 << 20,), float("nan"), device="cuda")     # (what a new tensor's memory may hold)
        del junk
        new = cache.attend(wide, SM, table, lens, q_starts=starts, max_q_len=3, **given)
        new, new_lse = new if isinstance(new, tuple) else (new, None)
        torch.cuda.synchronize()
        rest = torch.cat((new[:2], new[7:]))
        assert torch.equal(new[2:7], want) and (rest == (7 if "out" in given else 0)).all()
        if new_lse is not None:
            rest = torch.cat((new_lse[:2], new_lse[7:]))
            assert torch.equal(new_lse[2:7], lse[2:7])
            assert (rest == 5).all() if isinstance(given["lse"], torch.Tensor) else torch.isneginf(rest).all()


def test_rows_of_no_sequence_and_of_none_at_all():
    """Every workgroup clears its share: more rows than workgroups, around one short sequence, and no sequences."""
    cache = tkv.PagedCache(n_q_heads=4, n_kv_heads=2, n_pages=2)
    q = torch.randn(1500, 4, 128, device="cuda").half()
    starts = torch.tensor([700, 701], device="cuda", dtype=torch.int32)
    table, lens = torch.zeros(1, 1, device="cuda", dtype=torch.int32), torch.tensor([5], device="cuda", dtype=torch.int32)
    cache.v_pages[0, :, :5] = 3
    junk = torch.full((1 << 22,), float("nan"), device="cuda")
    del junk
    out, lse = cache.attend(q, SM, table, lens, q_starts=starts, max_q_len=1, lse=True)
    torch.cuda.synchronize()
    assert (out[700] == 3).all() and not out[:700].any() and not out[701:].any()
    assert lse[700].isfinite().all() and torch.isneginf(lse[:700]).all() and torch.isneginf(lse[701:]).all()
    out, lse = cache.attend(q[:3], SM, table[:0], lens[:0], q_starts=starts[:1] * 0, max_q_len=1, lse=True)
    torch.cuda.synchronize()
    assert not out.any() and torch.isneginf(lse).all()
    out = cache.attend(q[:0], SM, table[:0], lens[:0])
    assert tuple(out.shape) == (0, 4, 128)


@BOTH
def test_lengths_beyond_the_table_and_below_zero(bits):
    page = 32
    cache, q, table, lens, _ = _run([1, 1], [64, 96], 4, 1, page, bits, seed=9, starts=False)
    bad = torch.tensor([-5, 2**31 - 1], device="cuda", dtype=torch.int32)
    out, lse = cache.attend(q, SM, table, bad, lse=True)
    want = cache.attend(q, SM, table, lens)
    torch.cuda.synchronize()
    assert not out[0].any() and torch.isneginf(lse[0]).all()
    assert torch.equal(out[1], want[1])


@BOTH
def test_pages_outside_the_cache_stand_for_zeros(bits):
    page = 16
    pages, table, rows = _filled([80], 1, page, bits, torch.float16, seed=10)
    cache = tkv.PagedCache(n_q_heads=4, n_kv_heads=1, page_size=page, bits=bits, k_pages=pages[0], v_pages=pages[1])
    q = torch.randn(1, 4, 128, device="cuda").half()
    k, v = (x.copy() for x in rows[0])
    for place, bad in ((1, -1), (3, pages[0].shape[0])):
        table[0, place] = bad
        k[place * page:(place + 1) * page] = 0
        v[place * page:(place + 1) * page] = 0
    out, lse = cache.attend(q, SM, table, torch.tensor([80], device="cuda", dtype=torch.int32), lse=True)
    torch.cuda.synchronize()
    _compare(out, lse, _f64(q), k, v, torch.float16)


@BOTH
def test_pages_outside_the_cache_with_many_sixteens(bits):
    """Every sixteen of a page's tokens, not its first alone, and page 0, whose address stands in for that of none, holds numbers."""
    page = 64
    cache = tkv.PagedCache(n_q_heads=8, n_kv_heads=2, page_size=page, bits=bits, n_pages=6)
    k, v = (torch.randn(6 * page, 2, 128, device="cuda").half() for _ in range(2))
    slots = torch.arange(6 * page, device="cuda", dtype=torch.int32)
    cache.append(None, k, v, slots)
    k, v = (_f64(x) for x in cache.gather(slots))
    table = torch.tensor([[1, 6, 2, -3, 0]], device="cuda", dtype=torch.int32)
    kk, vv = (np.concatenate([x[p * page:(p + 1) * page] if 0 <= p < 6 else 0 * x[:page] for p in table[0].tolist()])[:300] for x in (k, v))
    q = torch.randn(1, 8, 128, device="cuda").half()
    out, lse = cache.attend(q, SM, table, torch.tensor([300], device="cuda", dtype=torch.int32), lse=True)
    torch.cuda.synchronize()
    _compare(out, lse, _f64(q), kk, vv, torch.float16)


def test_tables_without_pages():
    cache = tkv.PagedCache(n_q_heads=4, n_kv_heads=2, n_pages=2)
    q = torch.randn(3, 4, 128, device="cuda").half()
    table = torch.empty(3, 0, device="cuda", dtype=torch.int32)
    for n in (0, 5):
        out, lse = cache.attend(q, SM, table, torch.full((3,), n, device="cuda", dtype=torch.int32), lse=True)
        torch.cuda.synchronize()
        assert not out.any() and torch.isneginf(lse).all()


@BOTH
@pytest.mark.parametrize("hq,hkv", [(1024, 1), (1024, 1024), (1000, 8)])
def test_most_heads(hq, hkv, bits):
    print(f"case heads {hq}/{hkv} {bits} bits", flush=True)
    _run([1, 2], [65, 30], hq, hkv, 16, bits, seed=hkv)


@BOTH
def test_shared_pages(bits):
    """Sequences whose first pages are the same ones."""
    page = 16
    pages, table, rows = _filled([64, 40], 2, page, bits, torch.float16, seed=11)
    cache = tkv.PagedCache(n_q_heads=4, n_kv_heads=2, page_size=page, bits=bits, k_pages=pages[0], v_pages=pages[1])
    both = torch.cat((table, table[:1]))
    both[2, 2] = table[1, 0]                          # 32 tokens of the first, then 16 of the second
    q = torch.randn(3, 4, 128, device="cuda").half()
    out, lse = cache.attend(q, SM, both, torch.tensor([64, 40, 47], device="cuda", dtype=torch.int32), lse=True)
    torch.cuda.synchronize()
    k, v = (np.concatenate((rows[0][i][:32], rows[1][i][:15])) for i in range(2))
    for b, (kk, vv) in enumerate((rows[0], rows[1], (k, v))):
        _compare(out[b:b + 1], lse[b:b + 1], _f64(q[b:b + 1]), kk, vv, torch.float16)


@pytest.mark.parametrize("layout", ["tokens first", "both in one"])
def test_strides_of_pages(layout):
    hq, hkv, page, n_pages, dt = 8, 2, 32, 7, torch.float16
    if layout == "tokens first":
        k, v = (torch.randn(n_pages, page, hkv, 128, device="cuda").to(dt).transpose(1, 2) for _ in range(2))
    else:
        both = torch.randn(n_pages, 2, hkv, page, 128, device="cuda").to(dt)
        k, v = both[:, 0], both[:, 1]
    cache = tkv.PagedCache(n_q_heads=hq, n_kv_heads=hkv, page_size=page, k_pages=k, v_pages=v)
    table = torch.tensor([[5, 1, 0, 6]], device="cuda", dtype=torch.int32)
    q = torch.randn(1, hq, 128, device="cuda").to(dt)
    out, lse = cache.attend(q, SM, table, torch.tensor([123], device="cuda", dtype=torch.int32), lse=True)
    torch.cuda.synchronize()
    kk, vv = (_f64(x)[[5, 1, 0, 6]].transpose(0, 2, 1, 3).reshape(-1, hkv, 128)[:123] for x in (k, v))
    _compare(out, lse, _f64(q), kk, vv, dt)


@BOTH
def test_far_logits_and_large_values(bits):
    """Logits of thousands (one weight is all), and values near the type's largest."""
    page, dt = 32, torch.float16
    k = (60 * torch.randn(200, 1, 128, device="cuda")).to(dt)
    v = (20000 * torch.randn(200, 1, 128, device="cuda")).clamp(-60000, 60000).to(dt)
    cache = tkv.PagedCache(n_q_heads=4, n_kv_heads=1, page_size=page, bits=bits, n_pages=7)
    slots = torch.arange(200, device="cuda", dtype=torch.int32)
    cache.append(None, k, v, slots)
    k, v = cache.gather(slots)
    q = (30 * torch.randn(1, 4, 128, device="cuda")).to(dt)
    table = torch.arange(7, device="cuda", dtype=torch.int32)[None].contiguous()
    out = cache.attend(q, SM, table, torch.tensor([200], device="cuda", dtype=torch.int32))
    torch.cuda.synchronize()
    ref, _ = prompt_attention(_f64(q), _f64(k), _f64(v), SM)
    size, _ = prompt_attention(_f64(q), _f64(k), np.abs(_f64(v)), SM)
    # logits of magnitude up to 30 60 4 sqrt(128) sm ~ 1e4 have float32 errors of 1e4 2^-24 8: 5e-3 of a weight.  Where every value with
    # a weight is 0 (4 bits), what is left is absolute: half a step of fp16's smallest numbers, 2^-25, above all that 200 weights
    # below float32's smallest, 2^-126, add up to with values below 2^16 (2^-102).
    assert (np.abs(_f64(out) - ref) <= 2.0 ** -11 * np.abs(ref) + (1.1 * 2.0 ** -11 + 1e-2) * size + 2.0 ** -25).all()


@BOTH
def test_nan_in_a_seen_token_reaches_its_own_heads_only(bits):
    page = 16
    pages, table, rows = _filled([50, 60], 2, page, bits, torch.float16, seed=12)
    cache = tkv.PagedCache(n_q_heads=4, n_kv_heads=2, page_size=page, bits=bits, k_pages=pages[0], v_pages=pages[1])
    q = torch.randn(2, 4, 128, device="cuda").half()
    lens = torch.tensor([50, 60], device="cuda", dtype=torch.int32)
    want = cache.attend(q, SM, table, lens)
    bad = torch.full((1, 2, 128), 1.0, device="cuda").half()
    bad[0, 1, 5] = float("nan")
    slot = torch.from_numpy(paged.sequence_slots(table[1].cpu().numpy(), 60, page)[33:34].astype(np.int32)).cuda()
    cache.append(None, bad, torch.ones_like(bad), slot)
    out = cache.attend(q, SM, table, lens)
    torch.cuda.synchronize()
    assert torch.equal(out[0], want[0]) and out[1, 2:].isnan().all() and not out[1, :2].isnan().any()


@BOTH
def test_streams_threads_and_a_graph_over_a_growing_cache(bits):
    """A captured decode step (append, attend) replays while lengths, slots and positions move on; eager calls of the same object on
    another stream run beside it."""
    from test_gpu_rope import _freq
    page, hq, hkv, n_pages, b = 16, 8, 2, 12, 3
    cache = tkv.PagedCache(n_q_heads=hq, n_kv_heads=hkv, page_size=page, bits=bits, n_pages=n_pages)
    twin = tkv.PagedCache(n_q_heads=hq, n_kv_heads=hkv, page_size=page, bits=bits, n_pages=n_pages)
    table = torch.randperm(n_pages, generator=torch.Generator().manual_seed(0)).to(torch.int32).view(b, 4).cuda()
    f = _freq(128)
    rows = torch.randn(b, hq + 2 * hkv, 128, device="cuda").half()
    lens = torch.tensor([0, 20, 13], device="cuda", dtype=torch.int32)
    for c in (cache, twin):
        for i in range(b):
            n = int(lens[i])
            s = torch.from_numpy(paged.sequence_slots(table[i].cpu().numpy(), n, page).astype(np.int32)).cuda()
            g = torch.Generator(device="cuda").manual_seed(i)
            c.append(None, *(torch.randn(n, hkv, 128, generator=g, device="cuda").half() for _ in range(2)), s)

    def step(c):
        at = lens // page
        slots = (table.gather(1, at[:, None].long())[:, 0] * page + lens % page).to(torch.int32)
        q = c.append(rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:], slots, lens, f)
        return c.attend(q, SM, table, lens + 1, lse=True)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        caught = step(cache)
    side = torch.cuda.Stream()
    for i in range(6):
        graph.replay()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            want = step(twin)
            beside = cache.attend(rows[:, :hq].contiguous(), SM, table, lens)
        torch.cuda.synchronize()
        assert torch.equal(caught[0], want[0]) and torch.equal(caught[1], want[1]), i
        assert torch.equal(beside, cache.attend(rows[:, :hq].contiguous(), SM, table, lens))
        lens += torch.tensor([1, 3, 2], device="cuda", dtype=torch.int32)    # (some slots are skipped: zeros there)
        rows.mul_(0.9)


def test_prompt_then_chunk_then_decode():
    """As they are used: a prompt's rows normed, turned and put into 4-bit and 16-bit pages, a second chunk whose attention runs over the
    gathered prefix, decode steps over the pages; the pages' attention agrees with the prompt attention over the gathered rows."""
    from test_gpu_rope import _freq, _inputs
    hq, hkv, page, n1, n2 = 8, 2, 32, 150, 61
    f = _freq(128)
    q, k, v, qw, kw = _inputs(n1 + n2 + 4, hq, hkv, torch.bfloat16, seed=1)
    pos = torch.arange(n1 + n2 + 4, device="cuda", dtype=torch.int32)
    a = dict(norm=True, q_weight=qw, k_weight=kw)
    plan = tkv.PromptAttention(n_q_heads=hq, n_kv_heads=hkv)
    for bits in (16, 4):
        cache = tkv.PagedCache(n_q_heads=hq, n_kv_heads=hkv, page_size=page, bits=bits, n_pages=9)
        table = torch.tensor([[7, 0, 3, 8, 1, 5, 2]], device="cuda", dtype=torch.int32)
        slots = torch.from_numpy(paged.sequence_slots(table[0].cpu().numpy(), 224, page).astype(np.int32)).cuda()

        def put(i, j):
            return cache.append(q[i:j], k[i:j], v[i:j], slots[i:j], pos[i:j], f, **a)

        def from_rows(x, n):
            kk, vv = cache.gather(slots[:n])
            return plan.attend(x, kk, vv, SM, [len(x)], [n], lse=True)

        for i, j in ((0, n1), (n1, n1 + n2), *((n1 + n2 + s, n1 + n2 + s + 1) for s in range(4))):
            x = put(i, j)
            out, lse = cache.attend(x, SM, table, torch.tensor([j], device="cuda", dtype=torch.int32),
                                    q_starts=torch.tensor([0, j - i], device="cuda", dtype=torch.int32), max_q_len=j - i, lse=True)
            want, want_lse = from_rows(x, j)
            torch.cuda.synchronize()
            kk, vv = cache.gather(slots[:j])
            _compare(out, lse, _f64(x), _f64(kk), _f64(vv), torch.float16)
            assert (lse - want_lse).abs().max() <= 2e-5


@BOTH
def test_one_kv_head_and_a_long_sequence(bits):
    """More workgroups than an item's parts may be; rows of all kinds of joins."""
    for hq, n in ((4, 20011), (12, 30000), (32, 9999), (64, 5000)):
        print(f"case {hq}/1 heads over {n} {bits} bits", flush=True)
        _run([1], [n], hq, 1, 64, bits, seed=hq, starts=False)


@BOTH
def test_items_of_every_size_beside_each_other(bits):
    """Cuts at every place of an item: in its first tile, its last, at its beginning; workgroups in one item and in many."""
    rng = np.random.default_rng(3)
    for case in range(6):
        b = int(rng.integers(2, 90))
        lens = [int(n) for n in np.where(rng.random(b) < 0.2, rng.integers(500, 4000, b), rng.integers(0, 200, b))]
        q_lens = [int(n) for n in rng.integers(0, 4, b)]
        hq, hkv = [(8, 2), (8, 8), (16, 1), (6, 3)][case % 4]
        print(f"case mixed {case} {b} sequences {bits} bits", flush=True)
        _run(q_lens, lens, hq, hkv, 16, bits, seed=case)


@BOTH
def test_pools_beyond_4_gib(bits):
    """Pages at the far end of a pool of more than 2^32 bytes, and of more than 2^31 elements."""
    hkv, page = 8, 64
    n_pages = 40000 if bits == 16 else 135000          # 5.2 GB, 4.7 GB each of keys and values
    shape, dt = ((n_pages, hkv, page, 128), torch.float16) if bits == 16 else ((n_pages, hkv, 68 * page), torch.uint8)
    pages = [torch.empty(shape, dtype=dt, device="cuda") for _ in range(2)]
    cache = tkv.PagedCache(n_q_heads=16, n_kv_heads=hkv, page_size=page, bits=bits, k_pages=pages[0], v_pages=pages[1])
    n = 200
    table = torch.tensor([[n_pages - 1, 3, n_pages - 2, n_pages // 2 + 7]], dtype=torch.int32)
    slots = torch.from_numpy(paged.sequence_slots(table[0].numpy(), n, page).astype(np.int32)).cuda()
    k, v = (torch.randn(n, hkv, 128, device="cuda").half() for _ in range(2))
    cache.append(None, k, v, slots)
    got = cache.gather(slots)
    if bits == 16:
        assert torch.equal(got[0], k) and torch.equal(got[1], v)
    q = torch.randn(1, 16, 128, device="cuda").half()
    out, lse = cache.attend(q, SM, table.cuda(), torch.tensor([n], device="cuda", dtype=torch.int32), lse=True)
    torch.cuda.synchronize()
    _compare(out, lse, _f64(q), _f64(got[0]), _f64(got[1]), torch.float16)


def test_stream_with_compute_unit_mask():
    """On part of the machine there are fewer ranges."""
    import ctypes as C
    print("case masked stream", flush=True)
    hip = C.CDLL("libamdhip64.so")
    create = hip.hipExtStreamCreateWithCUMask
    create.argtypes = [C.POINTER(C.c_void_p), C.c_uint32, C.POINTER(C.c_uint32)]
    create.restype = C.c_int
    mask = (C.c_uint32 * 8)(0xFFFF0000, 0xFFFFFFFF, 0xFFFFFFFF, 0x0000FFFF, 0, 0, 0, 0)   # 96 units
    handle = C.c_void_p()
    if create(C.byref(handle), 8, mask) != 0 or not handle.value:
        pytest.skip("streams with a compute-unit mask are not available")
    try:
        for bits in (16, 4):
            pages, table, rows = _filled([3000, 700], 2, 32, bits, torch.float16, seed=13)
            cache = tkv.PagedCache(n_q_heads=8, n_kv_heads=2, page_size=32, bits=bits, k_pages=pages[0], v_pages=pages[1])
            q = torch.randn(2, 8, 128, device="cuda").half()
            lens = torch.tensor([3000, 700], device="cuda", dtype=torch.int32)
            torch.cuda.synchronize()
            out, lse = cache.attend(q, SM, table, lens, lse=True, stream=handle.value)
            again = cache.attend(q, SM, table, lens, stream=handle.value)
            torch.cuda.synchronize()
            assert torch.equal(out, again)
            for b, (k, v) in enumerate(rows):
                _compare(out[b:b + 1], lse[b:b + 1], _f64(q[b:b + 1]), k, v, torch.float16)
    finally:
        torch.cuda.synchronize()
        hip.hipStreamDestroy(handle)


def test_threads_with_streams_of_their_own_and_one_object():
    import threading
    lens = [[900, 33], [5, 2100]]
    made = [_filled(n, 2, 32, 16, torch.float16, seed=20 + i) for i, n in enumerate(lens)]
    pages = [torch.cat((made[0][0][i], made[1][0][i])) for i in range(2)]
    cache = tkv.PagedCache(n_q_heads=8, n_kv_heads=2, page_size=32, k_pages=pages[0], v_pages=pages[1])
    tables = [made[0][1], torch.where(made[1][1] < 10**6, made[1][1] + made[0][0][0].shape[0], made[1][1])]
    q = [torch.randn(2, 8, 128, device="cuda").half() for _ in range(2)]
    k_lens = [torch.tensor(n, device="cuda", dtype=torch.int32) for n in lens]
    want = [cache.attend(q[i], SM, tables[i], k_lens[i]) for i in range(2)]
    torch.cuda.synchronize()
    bad = []

    def work(i):
        torch.cuda.set_device(0)
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(50):
                if not torch.equal(cache.attend(q[i], SM, tables[i], k_lens[i]), want[i]):
                    bad.append(i)
            torch.cuda.current_stream().synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad
    for i in range(2):
        for b, (k, v) in enumerate(made[i][2]):
            ref, _ = prompt_attention(_f64(q[i][b:b + 1]), k, v, SM)
            assert np.abs(_f64(want[i][b:b + 1]) - ref).max() < 2e-3


def test_two_graphs_and_eager_calls_of_one_object():
    """Graphs captured from one object replay beside each other on streams of their own."""
    pages, table, rows = _filled([3000, 700], 2, 32, 16, torch.float16, seed=14)
    cache = tkv.PagedCache(n_q_heads=8, n_kv_heads=2, page_size=32, k_pages=pages[0], v_pages=pages[1])
    lens = torch.tensor([3000, 700], device="cuda", dtype=torch.int32)
    qs = [torch.randn(2, 8, 128, device="cuda").half() for _ in range(3)]
    want = [cache.attend(q, SM, table, lens, lse=True) for q in qs]
    graphs, outs = [], []
    for q in qs[:2]:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(cache.attend(q, SM, table, lens, lse=True))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(10):
        for o in outs:
            o[0].zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        eager = cache.attend(qs[2], SM, table, lens, lse=True)
        torch.cuda.synchronize()
        for got, w in zip((*outs, eager), want):
            assert torch.equal(got[0], w[0]) and torch.equal(got[1], w[1])


@BOTH
def test_parts_of_earlier_calls_do_not_matter_and_counters_end_at_zero(bits):
    """The workspace's parts may hold anything before a call, NaN and infinities included; its counters are 0 after every one."""
    lens = [3000, 700, 0, 20011, 33, 5000]
    print(f"case poisoned workspace {bits} bits", flush=True)
    cache, q, table, k_lens, want = _run([1] * 6, lens, 8, 2, 32, bits, seed=30, starts=False)
    workspace = list(cache._workspaces._of.values())[0]
    counters = workspace[-12288:]
    for i in range(30):
        workspace[:-12288].fill_((0xFF, 0x7C, 0x00)[i % 3])
        out = cache.attend(q, SM, table, k_lens)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and not counters.any(), i
