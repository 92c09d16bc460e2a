"""tkv_qk_norm_rope_axes, tkv_paged_append, tkv_paged_gather and tkv_paged_attn refuse what they cannot do before any GPU work (no GPU
needed)."""
import ctypes as C
import os

import pytest
import torch

import paper_2505_19586_amd as tkv
from paper_2505_19586_amd import build as tkv_build
from paper_2505_19586_amd.tkv import PagedDesc, RopeDesc

A = 4096  # an aligned address that is never read
INF = float("inf")


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(tkv.library_path()):
        tkv_build.build_library()
    return tkv.lib()


def _rope(**kw):
    d = RopeDesc(C.sizeof(RopeDesc), 32, 8, 128, 0, 0, 1, 1e-6, 128, 0, 6144, 128, 6144, 128, 6144, 128)
    for key, x in kw.items():
        setattr(d, key, x)
    return d


def _paged(**kw):
    d = PagedDesc(C.sizeof(PagedDesc), 32, 8, 128, 0, 16, 64, 100, (65536, 8192, 128), (65536, 8192, 128))
    for key, x in kw.items():
        setattr(d, key, (C.c_int64 * 3)(*x) if key.endswith("_stride") else x)
    return d


DESC = [
    (dict(struct_size=8), -1), (dict(n_q_heads=0), -1), (dict(n_kv_heads=-1), -1), (dict(n_q_heads=30), -1), (dict(head_dim=64), -2),
    (dict(head_dim=0), -1), (dict(n_q_heads=2048), -2), (dict(dtype=2), -1), (dict(bits=8), -2), (dict(page_size=0), -1),
    (dict(page_size=8), -2), (dict(page_size=48), -2), (dict(page_size=2048), -2), (dict(n_pages=0), -1), (dict(n_pages=1 << 25), -2),
    (dict(k_stride=(65536, 8192, 120)), -1), (dict(k_stride=(65536, 8192, 64)), -1), (dict(v_stride=(65536, 8192, 130)), -1),
    (dict(v_stride=(65528, 8192, 128)), -1), (dict(k_stride=(65536, 8184, 128)), -1), (dict(k_stride=(-65536, 8192, 128)), -1),
    (dict(k_stride=(0, 8192, 128)), -1), (dict(k_stride=(1 << 40, 8192, 128)), -1), (dict(v_stride=(1 << 34, 1 << 30, 1 << 23)), -1),
    (dict(v_stride=(65536, 128, 1024)), 0), (dict(k_stride=(131072, 16384, 256)), 0), (dict(bits=4, k_stride=(0, 0, 0)), 0),
    (dict(n_pages=(1 << 25) - 1), 0), (dict(n_kv_heads=1, k_stride=(65536, 0, 128)), 0), (dict(k_stride=(128, 819200, 12800)), 0),
]


@pytest.mark.parametrize("kw,status", DESC)
def test_descriptors(L, kw, status):
    n = C.c_size_t()
    assert L.tkv_paged_cache_sizes(C.byref(_paged(**kw)), C.byref(n)) == status
    assert L.tkv_paged_attn_sizes(C.byref(_paged(**kw)), C.byref(n)) == status
    if status:
        assert _append(L, desc=kw) == status and _gather(L, desc=kw) == status and _attn(L, desc=kw) == status


def test_sizes(L):
    n = C.c_size_t()
    assert L.tkv_paged_cache_sizes(C.byref(_paged()), C.byref(n)) == 0 and n.value == 100 * 8 * 64 * 256
    assert L.tkv_paged_cache_sizes(C.byref(_paged(bits=4)), C.byref(n)) == 0 and n.value == 100 * 8 * 64 * 68
    assert L.tkv_paged_cache_sizes(C.byref(_paged()), None) == -1 and L.tkv_paged_attn_sizes(C.byref(_paged()), None) == -1
    assert L.tkv_paged_cache_sizes(None, C.byref(n)) == -1 and L.tkv_paged_attn_sizes(None, C.byref(n)) == -1


def _axes(L, n=3, axis_of=bytes([0] * 24 + [1] * 20 + [2] * 20), n_axes=3, ptr=None, **kw):
    args = dict(q=A, k=A, v=A, positions=A, inv_freq=A, axis_of=axis_of, n_axes=n_axes, q_weight=A, k_weight=A, q_out=A, k_out=A, v_out=A)
    args.update(ptr or {})
    return L.tkv_qk_norm_rope_axes(C.byref(_rope(**kw)), n, *args.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(axis_of=None), -1), (dict(n_axes=2), -1), (dict(n_axes=0), -1), (dict(n_axes=-1), -1), (dict(n_axes=5), -2),
    (dict(axis_of=bytes([3] + [0] * 63)), -1), (dict(rotary_dim=24), -2), (dict(n=-1), -1), (dict(ptr=dict(positions=0)), -1),
    (dict(ptr=dict(q=0)), -1), (dict(ptr=dict(v=0)), -1), (dict(ptr=dict(q_out=A + 2)), -1), (dict(q_stride=6145), -1), (dict(n=0), 0),
    (dict(n=0, n_axes=2), -1), (dict(n=0, rotary_dim=32, n_axes=1), 0),
])
def test_axes(L, kw, status):
    assert _axes(L, **kw) == status


def _append(L, n=3, desc=None, ptr=None, axis_of=None, n_axes=1, **kw):
    args = dict(q=A, k=A, v=A, positions=A, inv_freq=A, axis_of=axis_of, n_axes=n_axes, q_weight=A, k_weight=A, slots=A, q_out=A, k_out=A,
                k_pages=A, v_pages=A)
    args.update(ptr or {})
    return L.tkv_paged_append(C.byref(_paged(**(desc or {}))), C.byref(_rope(**kw)), n, *args.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(desc=dict(n_q_heads=64)), -1), (dict(n_kv_heads=4), -1), (dict(out_dtype=1), -1), (dict(rotary_dim=40), -2), (dict(n=-2), -1),
    (dict(norm=0), -1), (dict(struct_size=0), -1), (dict(k_stride=6140), -1), (dict(v_stride=-8), -1),
    (dict(ptr=dict(k=0)), -1), (dict(ptr=dict(v=0)), -1), (dict(ptr=dict(slots=0)), -1), (dict(ptr=dict(k_pages=0)), -1),
    (dict(ptr=dict(v_pages=0)), -1), (dict(ptr=dict(q=0)), -1), (dict(ptr=dict(q_out=0)), -1), (dict(ptr=dict(q=0, q_out=0)), -1),
    (dict(ptr=dict(positions=0)), -1), (dict(ptr=dict(k_pages=A + 8)), -1), (dict(ptr=dict(k_out=A + 8)), -1), (dict(ptr=dict(slots=A + 2)), -1),
    (dict(axis_of=bytes([1] * 64)), -1), (dict(axis_of=bytes([1] * 64), n_axes=5), -2), (dict(n=0), 0), (dict(n=0, out_dtype=1), -1),
    (dict(n=(1 << 31) - 1), -2),
])
def test_append(L, kw, status):
    assert _append(L, **kw) == status


def _gather(L, n=3, desc=None, ptr=None):
    args = dict(k_pages=A, v_pages=A, n=n, slots=A, k_out=A, v_out=A)
    args.update(ptr or {})
    return L.tkv_paged_gather(C.byref(_paged(**(desc or {}))), *args.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), -1), (dict(n=0), 0), (dict(n=(1 << 31) - 1), -2), (dict(ptr=dict(k_pages=0)), -1), (dict(ptr=dict(v_pages=A + 4)), -1),
    (dict(ptr=dict(slots=0)), -1), (dict(ptr=dict(slots=A + 1)), -1), (dict(ptr=dict(k_out=0)), -1), (dict(ptr=dict(v_out=A + 8)), -1),
])
def test_gather(L, kw, status):
    assert _gather(L, **kw) == status


def _attn(L, desc=None, ptr=None, batch=3, n=3, most=1, each=7, scale=0.1, ws=1 << 40):
    args = dict(k_pages=A, v_pages=A, batch=batch, n=n, most=most, q=A, out=A, lse=A, table=A, each=each, k_lens=A, q_starts=0, clear=0, scale=scale,
                workspace=A, ws=ws)
    args.update(ptr or {})
    return L.tkv_paged_attn(C.byref(_paged(**(desc or {}))), *args.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(batch=-1), -1), (dict(n=-1), -1), (dict(n=4), -1), (dict(most=0), -1), (dict(most=2), -1), (dict(each=-1), -1),
    (dict(each=1 << 26), -2), (dict(each=(1 << 24) + 1), -2),
    (dict(each=1 << 24, ws=8), -4), (dict(batch=8, n=8, each=1 << 24), -2), (dict(batch=4000, n=4000, each=2048, ws=8), -4),
    (dict(n=1 << 23, most=1 << 23, ptr=dict(q_starts=A)), -2), (dict(desc=dict(n_q_heads=1024, n_kv_heads=1), n=4096, most=4096, ptr=dict(q_starts=A)), -2),
    (dict(desc=dict(n_q_heads=1024, n_kv_heads=1), n=4095, most=9999, ws=8, ptr=dict(q_starts=A)), -4), (dict(scale=0.0), -1), (dict(scale=-1.0), -1), (dict(scale=float("nan")), -1), (dict(scale=INF), -1),
    (dict(scale=3e38), -1), (dict(ws=8), -4), (dict(ptr=dict(workspace=0)), -1), (dict(ptr=dict(workspace=A + 4)), -1),
    (dict(ptr=dict(q=0)), -1), (dict(ptr=dict(q=A + 8)), -1), (dict(ptr=dict(out=0)), -1), (dict(ptr=dict(out=A + 2)), -1),
    (dict(ptr=dict(lse=A + 2)), -1), (dict(ptr=dict(table=0)), -1), (dict(ptr=dict(table=A + 1)), -1), (dict(ptr=dict(k_lens=0)), -1),
    (dict(ptr=dict(k_lens=A + 2)), -1), (dict(ptr=dict(q_starts=A + 2)), -1), (dict(ptr=dict(k_pages=0)), -1),
    (dict(ptr=dict(v_pages=A + 8)), -1), (dict(ptr=dict(clear=2)), -1), (dict(batch=0, n=0), 0), (dict(batch=0, n=5, ptr=dict(q_starts=A)), 0),
    (dict(n=0, ptr=dict(q_starts=A)), 0),
])
def test_attn(L, kw, status):
    assert _attn(L, **kw) == status


def test_null_descriptors(L):
    assert L.tkv_qk_norm_rope_axes(None, 1, A, A, A, A, A, bytes(64), 1, *([A] * 5), None) == -1
    assert L.tkv_paged_append(None, C.byref(_rope()), 1, *([A] * 5), None, 1, *([A] * 7), None) == -1
    assert L.tkv_paged_append(C.byref(_paged()), None, 1, *([A] * 5), None, 1, *([A] * 7), None) == -1
    assert L.tkv_paged_gather(None, A, A, 1, A, A, A, None) == -1
    assert L.tkv_paged_attn(None, A, A, 1, 1, 1, A, A, A, A, 1, A, None, 0, 0.1, A, 1 << 40, None) == -1


def test_axes_of_sections():
    assert tkv.rope_axes((2, 3, 1)) == bytes([0, 0, 1, 1, 1, 2])
    assert tkv.rope_axes((2, 3, 1), interleaved=True) == bytes([0, 1, 2, 0, 1, 1])
    for interleaved in (False, True):
        with pytest.raises(AssertionError):
            tkv.rope_axes((2, -1, 3), interleaved)


def test_tensors_of_the_host():
    """Refused as what is wrong, also where there is no GPU."""
    x = torch.zeros(2, 4, 128, dtype=torch.float16)
    with pytest.raises(AssertionError):
        tkv.qk_norm_rope(x, x, None, None)
    with pytest.raises(AssertionError):
        tkv.PagedCache(n_q_heads=4, n_kv_heads=4, page_size=16, k_pages=x.new_zeros(2, 4, 16, 128), v_pages=x.new_zeros(2, 4, 16, 128))


def test_strides_whose_span_leaves_64_bits(L):
    n = C.c_size_t()
    wide = dict(n_pages=(1 << 27) - 1, page_size=16, n_kv_heads=8)
    for strides, status in (((1 << 36, 1 << 33, 1 << 22), -1), ((1 << 33, 1 << 29, 1 << 22), 0)):
        assert L.tkv_paged_cache_sizes(C.byref(_paged(**wide, k_stride=strides, v_stride=strides)), C.byref(n)) == status
