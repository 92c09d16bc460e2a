"""tkv_paged_append and tkv_paged_gather: what pages hold, bit for bit.  Rows of 16 bits are those of qk_norm_rope (whose own tests hold
them against float64), 4-bit blocks those that the oracle makes of them."""
import numpy as np
import pytest
import torch

import paper_2505_19586_amd as tkv
from oracle import paged
from test_gpu_rope import _freq, _inputs

pytestmark = pytest.mark.gpu
NAME = {torch.float16: "fp16", torch.bfloat16: "bf16"}


def _f64(x):
    return x.double().cpu().numpy()


def _slots(t, n_pages, page, seed=0):
    g = torch.Generator().manual_seed(seed)
    return torch.randperm(n_pages * page, generator=g)[:t].to(torch.int32).cuda()


def _pages(n_pages, hkv, page, bits, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if bits == 16:
        return [torch.randn(n_pages, hkv, page, 128, generator=g, device="cuda").to(dtype) for _ in range(2)]
    return [torch.randint(0, 256, (n_pages, hkv, 68 * page), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2)]


def _cache(hq, hkv, page, bits, dtype, k, v):
    return tkv.PagedCache(n_q_heads=hq, n_kv_heads=hkv, page_size=page, bits=bits, dtype=dtype, k_pages=k, v_pages=v)


def _holds(pages, before, rows, slots, page, dtype):
    """pages hold rows [T, Hkv, 128] at slots and what they held before elsewhere."""
    n = pages.shape[0] * page
    slots = slots.cpu().numpy()
    if pages.dtype != torch.uint8:
        want = before.clone()
        for t, s in enumerate(slots):
            if 0 <= s < n:
                want[s // page, :, s % page] = rows[t]
        assert torch.equal(pages.view(torch.int16), want.view(torch.int16))
        return
    want = before.cpu().numpy().copy()
    codes, scales = paged.split_page(want, page)   # (of the copy: written through below)
    x = _f64(rows)
    for t, s in enumerate(slots):
        if 0 <= s < n:
            for h in range(x.shape[1]):
                c, e = paged.encode_row(x[t, h], NAME[dtype])
                want[s // page, h, 64 * (s % page):64 * (s % page) + 64] = c
                want[s // page, h, 64 * page + 4 * (s % page):64 * page + 4 * (s % page) + 4] = e
    got = pages.cpu().numpy()
    # a zero's sign does not matter
    at = np.arange(want.shape[2]) < 64 * page
    low = lambda c: np.where(c & 15 == 8, c & 0xF0, c)  # noqa: E731
    high = lambda c: np.where(c >> 4 == 8, c & 0x0F, c)  # noqa: E731
    assert np.array_equal(np.where(at, low(high(got)), got), np.where(at, low(high(want)), want))


@pytest.mark.parametrize("src,dst", [(torch.float16, torch.float16), (torch.bfloat16, torch.float16), (torch.bfloat16, torch.bfloat16),
                                     (torch.float16, torch.bfloat16)])
@pytest.mark.parametrize("rot,interleaved", [(128, False), (128, True), (96, False), (64, False), (32, True), (16, False), (0, False)])
@pytest.mark.parametrize("bits", [16, 4])
def test_rows_in_their_slots(src, dst, rot, interleaved, bits):
    t, hq, hkv, page = 21, 5, 1, 16
    q, k, v, qw, kw = _inputs(t, hq, hkv, src)
    pos = torch.randint(0, 131072, (t,), device="cuda", dtype=torch.int32)
    f = _freq(rot)
    a = dict(norm=True, q_weight=qw, k_weight=kw, interleaved=interleaved)
    want = tkv.qk_norm_rope(q, k, pos, f, v=v, out_dtype=dst, **a)
    before = _pages(4, hkv, page, bits, dst)
    cache = _cache(hq, hkv, page, bits, dst, *[x.clone() for x in before])
    slots = _slots(t, 4, page)
    slots[3], slots[9], slots[20] = -1, 4 * page, 2**31 - 1          # padding
    k_out = torch.empty(t, hkv, 128, dtype=dst, device="cuda")
    got = cache.append(q, k, v, slots, pos, f, k_out=k_out, **a)
    assert torch.equal(got, want[0]) and torch.equal(k_out, want[1])
    _holds(cache.k_pages, before[0], want[1], slots, page, dst)
    _holds(cache.v_pages, before[1], want[2], slots, page, dst)


@pytest.mark.parametrize("page", [16, 32, 64, 256, 1024])
@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("hq,hkv", [(32, 8), (3, 3)])
def test_page_sizes_heads_and_axes(page, bits, hq, hkv):
    t = 150
    q, k, v, _, kw = _inputs(t, hq, hkv, torch.float16, seed=page)
    pos = torch.randint(0, 5000, (3, t), device="cuda", dtype=torch.int32)
    a = dict(axis_of=tkv.rope_axes((16, 24, 24)), norm=True, k_weight=kw, eps=1e-5)
    want = tkv.qk_norm_rope(q, k, pos, _freq(128), v=v, **a)
    n_pages = 3 if page >= 64 else 11
    before = _pages(n_pages, hkv, page, bits, torch.float16, 1)
    cache = _cache(hq, hkv, page, bits, torch.float16, *[x.clone() for x in before])
    slots = _slots(t, n_pages, page, page)
    assert torch.equal(cache.append(q, k, v, slots, pos, _freq(128), **a), want[0])
    _holds(cache.k_pages, before[0], want[1], slots, page, torch.float16)
    _holds(cache.v_pages, before[1], want[2], slots, page, torch.float16)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_every_number_of_the_type_in_4_bits(dtype):
    """Blocks of every bit pattern (subnormal numbers, infinities and NaN among them), each beside a larger one that sets the block's
    scale up to eight powers of two above it, and the same as the largest."""
    bits = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(dtype)
    rng = np.random.default_rng(2)
    rows = []
    x = bits.view(-1, 128).cuda()                                      # neighbours: their scale is their own
    rows.append(x)
    finite = bits[torch.isfinite(bits.float())]
    y = finite[torch.from_numpy(rng.permutation(finite.numel()))].clone()
    y = y[:y.numel() // 31 * 31].view(-1, 31)
    top = (y.float().abs().amax(1).clamp(min=float(torch.finfo(dtype).tiny)) * torch.from_numpy(2.0 ** rng.uniform(0, 8, y.shape[0])).float())
    z = torch.cat((y, top.clamp(max=float(torch.finfo(dtype).max)).to(dtype)[:, None]), 1)
    z = z[:z.shape[0] // 4 * 4].reshape(-1, 128).cuda()
    # one number of every magnitude among others up to eight powers of two larger
    rows.append(z)
    w = (torch.randn(300, 128, device="cuda") * 2.0 ** torch.randint(-14, 14, (300, 1), device="cuda")).to(dtype)
    rows.append(w)
    rows = torch.cat(rows)[:, None].contiguous()                       # [T, 1, 128]
    t = rows.shape[0]
    n_pages = -(-t // 64)
    cache = tkv.PagedCache(n_q_heads=1, n_kv_heads=1, bits=4, dtype=dtype, n_pages=n_pages)
    slots = torch.arange(t, device="cuda", dtype=torch.int32)
    other = rows.flip(0).contiguous()
    assert cache.append(None, rows, other, slots) is None
    k, v = cache.gather(slots)
    codes, scales = zip(*(paged.encode_row(r, NAME[dtype]) for r in _f64(rows[:, 0])))
    codes, scales = np.array(codes), np.array(scales)
    got_codes, got_scales = paged.split_page(cache.k_pages.cpu().numpy()[:, 0], 64)
    assert np.array_equal(got_scales.reshape(-1, 4)[:t], scales)
    held = paged.decode_rows(got_codes.reshape(-1, 64)[:t], scales)
    want = paged.decode_rows(codes, scales)
    assert np.array_equal(held, want, equal_nan=True)
    assert np.array_equal(_f64(k)[:, 0], want, equal_nan=True)         # exact in the type
    assert np.array_equal(_f64(v)[::-1, 0], want, equal_nan=True)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("t", [1, 15, 16, 17, 333])
def test_gather(bits, dtype, t):
    page, hkv, n_pages = 32, 3, 9
    k, v = _pages(n_pages, hkv, page, bits, dtype, t)
    if bits == 4:
        for x in (k, v):   # scales whose blocks are numbers of the type, some NaN
            x[..., 64 * page:] = torch.randint(104, 140, x[..., 64 * page:].shape, device="cuda", dtype=torch.uint8)
            x[1, 0, 64 * page + 5] = 255
    cache = _cache(3, hkv, page, bits, dtype, k, v)
    g = torch.Generator().manual_seed(t)
    slots = torch.randint(0, n_pages * page, (t,), generator=g).to(torch.int32)
    slots[0] = page + 1
    if t > 4:
        slots[1], slots[2], slots[3] = -1, n_pages * page, -2**31       # zeros
        slots[4] = slots[0]                                             # the same twice
    got = cache.gather(slots.cuda())
    for x, pages in zip(got, (k, v)):
        pages = pages.cpu().numpy() if bits == 4 else _f64(pages)
        assert x.is_contiguous() and np.array_equal(_f64(x), paged.rows_of(pages, page, slots.tolist()), equal_nan=True)
    given = [torch.full_like(x, 3) for x in got]
    again = cache.gather(slots.cuda(), k_out=given[0], v_out=given[1])
    assert again[0] is given[0] and all(torch.equal(x.view(torch.int16), y.view(torch.int16)) for x, y in zip(again, got))


@pytest.mark.parametrize("layout", ["tokens first", "both in one", "wider rows"])
def test_strides_of_pages(layout):
    hq, hkv, page, n_pages, t, dt = 8, 2, 32, 5, 70, torch.bfloat16
    if layout == "tokens first":
        k, v = (torch.randn(n_pages, page, hkv, 128, device="cuda").to(dt).transpose(1, 2) for _ in range(2))
    elif layout == "both in one":
        both = torch.randn(n_pages, 2, hkv, page, 128, device="cuda").to(dt)
        k, v = both[:, 0], both[:, 1]
    else:
        wide = torch.randn(n_pages + 2, hkv + 1, page, 256, device="cuda").to(dt)
        k, v = wide[:n_pages, :hkv, :, :128], wide[2:, 1:, :, 128:]
    q, kn, vn, _, _ = _inputs(t, hq, hkv, dt)
    pos, f = torch.arange(t, device="cuda", dtype=torch.int32), _freq(128)
    slots = _slots(t, n_pages, page)
    before = [k.clone(), v.clone()]
    cache = _cache(hq, hkv, page, 16, dt, k, v)
    cache.append(q, kn, vn, slots, pos, f)
    want = tkv.qk_norm_rope(q, kn, pos, f, v=vn)
    for pages, old, rows in ((k, before[0], want[1]), (v, before[1], want[2])):
        _holds(pages.contiguous(), old.contiguous(), rows, slots, page, dt)
    got = cache.gather(slots)
    assert torch.equal(got[0], want[1]) and torch.equal(got[1], want[2])


def test_long_appends_and_replayed_graph():
    """Enough rows for waves of two octets; then a step that is captured and replayed with slots and positions that move on."""
    dt, page = torch.float16, 64
    for bits in (16, 4):
        q, k, v, qw, kw = _inputs(2000, 32, 4, torch.bfloat16, seed=bits)
        a = dict(norm=True, q_weight=qw, k_weight=kw)
        f = _freq(128)
        cache = tkv.PagedCache(n_kv_heads=4, bits=bits, page_size=page, n_pages=40, dtype=dt)
        short = tkv.PagedCache(n_kv_heads=4, bits=bits, page_size=page, n_pages=40, dtype=dt)
        pos, slots = torch.arange(2000, device="cuda", dtype=torch.int32), _slots(2000, 40, page, 1)
        got = cache.append(q, k, v, slots, pos, f, **a)
        parts = [short.append(q[i:i + 50], k[i:i + 50], v[i:i + 50], slots[i:i + 50], pos[i:i + 50], f, **a) for i in range(0, 2000, 50)]
        assert torch.equal(got, torch.cat(parts))
        assert torch.equal(cache.k_pages.view(torch.uint8), short.k_pages.view(torch.uint8))
        assert torch.equal(cache.v_pages.view(torch.uint8), short.v_pages.view(torch.uint8))

        step = dict(slots=slots[:9].clone(), positions=pos[:9].clone())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            caught = cache.append(q[:9], k[:9], v[:9], inv_freq=f, **step, **a)
            back = cache.gather(step["slots"])
        for i in range(4):
            step["slots"].copy_(slots[100 * i:100 * i + 9])
            step["positions"] += 7
            graph.replay()
            torch.cuda.synchronize()
            want = short.append(q[:9], k[:9], v[:9], inv_freq=f, **step, **a)
            rows = short.gather(step["slots"])
            assert torch.equal(caught, want) and all(torch.equal(x, y) for x, y in zip(back, rows))


def test_no_tokens():
    cache = tkv.PagedCache(n_pages=2)
    q, k, v, _, _ = _inputs(0, 32, 8, torch.float16)
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert tuple(cache.append(q, k, v, none, none, _freq(128)).shape) == (0, 32, 128)
    assert [tuple(x.shape) for x in cache.gather(none)] == [(0, 8, 128)] * 2
