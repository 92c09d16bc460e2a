"""tkv_prompt_attn refuses what it cannot do before any GPU work (no GPU needed), and the oracle of its tests."""
import ctypes as C
import os

import numpy as np
import pytest

import paper_2505_19586_amd as tkv
from oracle.attention import decode_attention
from oracle.prompt import prompt_attention
from paper_2505_19586_amd import build as tkv_build
from paper_2505_19586_amd.tkv import PromptDesc

A = 4096  # an aligned address that is never read


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(tkv.library_path()):
        tkv_build.build_library()
    return tkv.lib()


def _desc(**kw):
    d = PromptDesc(C.sizeof(PromptDesc), 32, 8, 128, 0, 1, 2, 0, (C.c_int64 * 8)(4096, 128, 1024, 128, 1024, 128, 4096, 128))
    for key, x in kw.items():
        if key.endswith("_stride"):
            i = 2 * "qkvo".index(key[0])
            d.strides[i], d.strides[i + 1] = x
        else:
            setattr(d, key, x)
    return d


def _call(L, lens=((0, 5), (5, 5), (0, 5), (5, 5)), ptr=None, sm=0.1, ws=1 << 30, **kw):
    d = _desc(**kw)
    arrays = [None if x is None else (C.c_int32 * 2)(*x) for x in lens]  # q_start, q_len, k_start, k_len
    p = dict(q=A, k=A, v=A, out=A, lse=A, ws=A)
    p.update(ptr or {})
    return L.tkv_prompt_attn(C.byref(d), p["q"], p["k"], p["v"], p["out"], p["lse"], *arrays, sm, p["ws"], ws, None)


@pytest.mark.parametrize("kw,status", [
    (dict(struct_size=4), -1), (dict(n_q_heads=30), -1), (dict(n_kv_heads=0), -1), (dict(head_dim=96), -2), (dict(dtype=2), -1),
    (dict(causal=2), -1), (dict(batch=0), -1), (dict(batch=65), -2), (dict(n_q_heads=2048), -2),
    (dict(q_stride=(4097, 128)), -1), (dict(k_stride=(1024, 12)), -1), (dict(v_stride=(-1024, 128)), -1),
    (dict(o_stride=(1 << 23, 128)), -1), (dict(sm=0.0), -1), (dict(sm=-1.0), -1), (dict(sm=float("nan")), -1),
    (dict(sm=float("inf")), -1), (dict(ws=1 << 20), -4), (dict(ptr=dict(ws=0)), -1), (dict(ptr=dict(q=0)), -1),
    (dict(ptr=dict(k=0)), -1), (dict(ptr=dict(out=0)), -1), (dict(ptr=dict(v=A + 8)), -1), (dict(ptr=dict(lse=A + 2)), -1),
    (dict(lens=((0, 5), (5, -1), (0, 5), (5, 5))), -1), (dict(lens=((0, -5), (5, 1), (0, 5), (5, 5))), -1),
    (dict(lens=((0, 5), (5, 5), (0, 5), None)), -1), (dict(lens=((0, 5), (1 << 30, 5), (0, 5), (5, 5))), -2),
    (dict(lens=((0, 2147483000), (5, 1000), (0, 5), (5, 5))), -1), (dict(lens=((0, 0), (0, 0), (0, 0), (5, 5))), 0),
])
def test_refusals(L, kw, status):
    assert _call(L, **kw) == status


@pytest.mark.parametrize("starts,lens,status", [
    ((0, 4), (5, 5), -1), ((4, 0), (5, 5), -1), ((3, 3), (1, 1), -1), ((0, 2), (5, 1), -1), ((2, 0), (1, 5), -1),
])
def test_no_row_belongs_to_two_sequences(L, starts, lens, status):
    assert _call(L, lens=(starts, lens, (0, 5), (5, 5))) == status


def test_more_rows_than_a_launch_has_workgroups(L):
    assert _call(L, lens=((0, 1 << 29), (1 << 27, 5), (0, 5), (5, 5)), n_q_heads=64, n_kv_heads=64) == -2


def test_sizes(L):
    n = C.c_size_t()
    assert L.tkv_prompt_attn_sizes(C.byref(_desc()), C.byref(n)) == 0 and n.value > 0
    assert L.tkv_prompt_attn_sizes(C.byref(_desc()), None) == -1
    assert L.tkv_prompt_attn_sizes(None, C.byref(n)) == -1
    assert L.tkv_prompt_attn_sizes(C.byref(_desc(dtype=5)), C.byref(n)) == -1


def test_oracle_by_hand_and_against_the_decode_oracle():
    v = np.array([1.0, 2.0, 4.0]).reshape(3, 1, 1) * np.ones((3, 1, 2))
    out, lse = prompt_attention(np.zeros((2, 1, 2)), np.zeros((3, 1, 2)), v, 1.0)    # equal weights: means of 2 and of 3 rows
    assert np.allclose(out[:, 0, 0], [1.5, 7 / 3]) and np.allclose(lse[:, 0], np.log([2, 3]))
    out, lse = prompt_attention(np.zeros((2, 1, 2)), np.zeros((1, 1, 2)), v[:1], 1.0)
    assert (out[0] == 0).all() and lse[0, 0] == -np.inf and (out[1] == 1).all()
    r = np.random.default_rng(1)
    q, k, v = r.standard_normal((5, 4, 16)), r.standard_normal((9, 2, 16)), r.standard_normal((9, 2, 16))
    out, _ = prompt_attention(q, k, v, 0.3)
    for i in range(5):
        assert np.allclose(out[i], decode_attention(q[i], k[:5 + i].transpose(1, 0, 2), v[:5 + i].transpose(1, 0, 2), 0.3))
    full, _ = prompt_attention(q, k, v, 0.3, causal=False)
    assert np.allclose(full[4], out[4]) and not np.allclose(full[0], out[0])
