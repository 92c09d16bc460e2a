"""tkv_quant_attn_decode_shared refuses what it cannot do before any GPU work (no GPU needed)."""
import ctypes as C
import os

import pytest

import paper_2505_19586_amd as tkv
from paper_2505_19586_amd import build as tkv_build
from paper_2505_19586_amd.tkv import QuantCache, QuantDesc

A = 4096  # an aligned address that is never read


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(tkv.library_path()):
        tkv_build.build_library()
    return tkv.lib()


def _desc(batch, **kw):
    d = QuantDesc(C.sizeof(QuantDesc), 32, 8, 128, 2, 32, 128, 4096, batch)
    for key, x in kw.items():
        setattr(d, key, x)
    return d


def _call(L, prefix=None, own=None, prefix_lens=(100, 4096), lens=(5, 0, 7), of=(0, 1, -1), ptr=None, sm=0.1, ws=1 << 30, cache=None):
    pd, d = _desc(2, **(prefix or {})), _desc(3, **(own or {}))
    p = dict(q=A, out=A, ws=A)
    p.update(ptr or {})
    pl, ol = (C.c_int32 * 2)(*prefix_lens), (C.c_int32 * 3)(*lens)
    pc, oc = QuantCache(*([A] * 8), pl), QuantCache(*([A] * 8), ol)
    for key, x in (cache or {}).items():
        setattr(oc, key, x)
    of = None if of is None else (C.c_int32 * 3)(*of)
    return L.tkv_quant_attn_decode_shared(C.byref(pd), C.byref(pc), C.byref(d), C.byref(oc), of, p["q"], p["out"], sm, p["ws"], ws, None)


@pytest.mark.parametrize("kw,status", [
    (dict(prefix=dict(struct_size=1)), -1), (dict(own=dict(bits=3)), -2), (dict(own=dict(bits=4)), -1),
    (dict(prefix=dict(group_size=64)), -1), (dict(own=dict(n_q_heads=64)), -1), (dict(prefix=dict(n_kv_heads=4)), -1),
    (dict(own=dict(head_dim=64)), -2), (dict(prefix_lens=(100, 4097)), -1), (dict(lens=(5, -1, 0)), -1),
    (dict(of=(0, 2, 0)), -1), (dict(of=(0, -2, 0)), -1), (dict(sm=0.0), -1), (dict(sm=float("nan")), -1), (dict(sm=float("inf")), -1),
    (dict(ws=1000), -4), (dict(ptr=dict(ws=0)), -1), (dict(ptr=dict(ws=A + 4)), -1), (dict(ptr=dict(q=A + 2)), -1),
    (dict(ptr=dict(q=0)), -1), (dict(ptr=dict(out=0)), -1), (dict(ptr=dict(out=A + 2)), -1), (dict(cache=dict(k_codes=0)), -1),
    (dict(cache=dict(v_zero=A + 2)), -1), (dict(cache=dict(seq_len_host=None)), -1),
])
def test_refusals(L, kw, status):
    assert _call(L, **kw) == status


def test_sizes_and_null_pointers(L):
    n = C.c_size_t()
    size = L.tkv_quant_attn_decode_shared_sizes
    assert size(C.byref(_desc(2)), C.byref(_desc(64)), C.byref(n)) == 0 and 0 < n.value < 32 << 20
    assert size(C.byref(_desc(2)), C.byref(_desc(64)), None) == -1
    assert size(None, C.byref(_desc(1)), C.byref(n)) == -1
    assert size(C.byref(_desc(2)), C.byref(_desc(2, bits=1)), C.byref(n)) == -1
    assert L.tkv_quant_attn_decode_shared(C.byref(_desc(1)), None, C.byref(_desc(1)), None, None, A, A, 0.1, A, 1 << 30, None) == -1
