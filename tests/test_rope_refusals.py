"""tkv_qk_norm_rope refuses what it cannot do before any GPU work (no GPU needed)."""
import ctypes as C
import os

import pytest

import paper_2505_19586_amd as tkv
from paper_2505_19586_amd import build as tkv_build
from paper_2505_19586_amd.tkv import RopeDesc

A = 4096  # an aligned address that is never read


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(tkv.library_path()):
        tkv_build.build_library()
    return tkv.lib()


def _call(L, n=3, ptr=None, **kw):
    d = RopeDesc(C.sizeof(RopeDesc), 32, 8, 128, 0, 0, 1, 1e-6, 128, 0, 6144, 128, 6144, 128, 6144, 128)
    for key, x in kw.items():
        if key.endswith("_stride"):
            setattr(d, key + "_head", x[1])
            x = x[0]
        setattr(d, key, x)
    args = dict(q=A, k=A, v=A, positions=A, inv_freq=A, q_weight=A, k_weight=A, q_out=A, k_out=A, v_out=A)
    args.update(ptr or {})
    return L.tkv_qk_norm_rope(C.byref(d), n, *args.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(struct_size=8), -1), (dict(n_q_heads=0), -1), (dict(n_kv_heads=-1), -1), (dict(head_dim=64), -2), (dict(head_dim=0), -1),
    (dict(n_q_heads=2000), -2), (dict(in_dtype=2), -1), (dict(out_dtype=-1), -1), (dict(norm=2), -1), (dict(norm=0), -1),
    (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1), (dict(rotary_dim=130), -1), (dict(rotary_dim=-16), -1),
    (dict(rotary_dim=17), -1), (dict(rotary_dim=24), -2), (dict(interleaved=3), -1), (dict(q_stride=(6145, 128)), -1),
    (dict(k_stride=(6144, 4)), -1), (dict(v_stride=(-8, 128)), -1), (dict(n=-1), -1),
    (dict(ptr=dict(q=0)), -1), (dict(ptr=dict(k_out=0)), -1), (dict(ptr=dict(v=0)), -1), (dict(ptr=dict(v_out=0)), -1),
    (dict(ptr=dict(positions=0)), -1), (dict(ptr=dict(inv_freq=0)), -1), (dict(ptr=dict(q=A + 2)), -1),
    (dict(ptr=dict(v_out=A + 8)), -1), (dict(ptr=dict(k_weight=A + 4)), -1), (dict(n=0), 0),
])
def test_refusals(L, kw, status):
    assert _call(L, **kw) == status


def test_more_tokens_than_a_launch_has_waves(L):
    assert _call(L, n=(1 << 31) - 1, n_q_heads=1, n_kv_heads=1) == -2


def test_null_descriptor(L):
    assert L.tkv_qk_norm_rope(None, 1, *([A] * 10), None) == -1
