"""tkv_qk_norm_rope against float64: types, pairings, partial rotation, far and negative positions, slices of a fused
projection, rows of zeros, outputs over their inputs, other streams and replayed graphs.

Tolerance: half a step of the output's type, and float32's errors relative to |a| + |b| of the channel's pair: the angle
rounded to 32 bits in half turns (pi 2^-25), sine and cosine (2^-23), 19 additions and the square root of the norm (10 2^-24),
five products and sums (5 2^-24): below 2^-19 together."""
import numpy as np
import pytest
import torch

import paper_2505_19586_amd as tkv
from oracle.rope import norm_rope

pytestmark = pytest.mark.gpu
F32 = 2.0 ** -19


def _freq(rot, dev="cuda"):
    return (500000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float().to(dev) if rot else None


def _check(got, x, pos, freq, dtype, **kw):
    ref, size = norm_rope(x.double().cpu().numpy(), None if pos is None else pos.cpu().numpy(),
                          None if freq is None else freq.cpu().numpy(), **kw)
    o = got.double().cpu().numpy()
    tiny = 2.0 ** -25 if dtype == torch.float16 else 0.0   # half the step of fp16's smallest numbers
    assert (np.abs(o - ref) <= torch.finfo(dtype).eps / 2 * np.abs(ref) + F32 * size + tiny).all()


def _inputs(t, hq, hkv, src, seed=0, fused=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows = torch.randn(t, hq + 2 * hkv, 128, generator=g, device="cuda").to(src)
    q, k, v = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
    w = [(1 + 0.3 * torch.randn(128, generator=g, device="cuda")).to(src) for _ in range(2)]
    return (q, k, v, *w) if fused else (q.contiguous(), k.contiguous(), v.contiguous(), *w)


@pytest.mark.parametrize("src,dst", [(torch.float16, torch.float16), (torch.bfloat16, torch.float16),
                                     (torch.bfloat16, torch.bfloat16), (torch.float16, torch.bfloat16)])
@pytest.mark.parametrize("rot,interleaved", [(128, False), (128, True), (96, False), (32, True), (16, False), (0, False)])
@pytest.mark.parametrize("norm", [False, True])
def test_types_and_pairings(src, dst, rot, interleaved, norm):
    q, k, v, qw, kw = _inputs(37, 5, 1, src)     # 7 rows of a token: no whole number of octets
    pos = torch.randint(0, 131072, (37,), device="cuda", dtype=torch.int32)
    f = _freq(rot)
    a = dict(norm=norm, q_weight=qw if norm else None, k_weight=kw if norm else None, interleaved=interleaved)
    oq, ok, ov = tkv.qk_norm_rope(q, k, pos, f, v=v, out_dtype=dst, **a)
    cpu = lambda w: None if w is None else w.double().cpu().numpy()  # noqa: E731
    for o, x, w in ((oq, q, a["q_weight"]), (ok, k, a["k_weight"])):
        assert o.dtype == dst and o.is_contiguous()
        _check(o, x, pos, f, dst, norm=norm, weight=cpu(w), interleaved=interleaved)
    assert torch.equal(ov, v.to(dst))


@pytest.mark.parametrize("t", [1, 2, 63, 4095, 4096, 5001])
@pytest.mark.parametrize("hq,hkv", [(32, 8), (64, 8), (1, 1)])
def test_lengths_and_heads(t, hq, hkv):
    q, k, _, qw, _ = _inputs(t, hq, hkv, torch.float16, seed=t, fused=t % 2 == 1)
    pos = torch.arange(t, device="cuda", dtype=torch.int32) + 126000
    f = _freq(128)
    oq, ok, ov = tkv.qk_norm_rope(q, k, pos, f, norm=True, q_weight=qw, eps=1e-5)
    assert ov is None
    some = slice(None) if t < 100 else [0, 1, t // 2, t - 2, t - 1]
    _check(oq[some], q[some], pos[some], f, torch.float16, norm=True, weight=qw.double().cpu().numpy(), eps=1e-5)
    _check(ok[some], k[some], pos[some], f, torch.float16, norm=True, eps=1e-5)
    # every row, against the same token in a call of its own kind of launch
    lone = tkv.qk_norm_rope(q[t - 1:], k[t - 1:], pos[t - 1:], f, norm=True, q_weight=qw, eps=1e-5)
    assert torch.equal(lone[0], oq[t - 1:]) and torch.equal(lone[1], ok[t - 1:])


def test_positions_of_any_sign_and_size():
    q, k, _, _, _ = _inputs(6, 2, 1, torch.float16)
    pos = torch.tensor([0, -1, -131072, 1 << 20, 2**31 - 1, -2**31], device="cuda", dtype=torch.int32)
    f = _freq(128)
    oq, ok, _ = tkv.qk_norm_rope(q, k, pos, f)
    # the float64 reference's own angle is off by 2^31 2^-53
    _check(oq, q, pos, f, torch.float16)
    _check(ok, k, pos, f, torch.float16)
    assert torch.equal(oq[0], q[0])          # position 0 turns nothing


def test_rows_of_zeros_and_non_finite_rows():
    q, k, _, _, _ = _inputs(4, 2, 1, torch.float16, fused=False)
    q[1] = 0
    q[2, 0, 5] = float("nan")
    q[3, 1, 5] = float("inf")
    pos, f = torch.arange(4, device="cuda", dtype=torch.int32), _freq(128)
    oq, ok, _ = tkv.qk_norm_rope(q, k, pos, f, norm=True)
    assert (oq[1] == 0).all()
    assert oq[2, 0].isnan().all() and not oq[2, 1].isnan().any() and not oq[3, 0].isnan().any()
    _check(ok, k, pos, f, torch.float16, norm=True)


def test_outputs_over_their_inputs_and_heads_in_another_order():
    q, k, v, qw, kw = _inputs(70, 32, 8, torch.bfloat16, fused=False)
    pos, f = torch.arange(70, device="cuda", dtype=torch.int32), _freq(128)
    want = tkv.qk_norm_rope(q, k, pos, f, v=v, norm=True, q_weight=qw, k_weight=kw)
    by_head = q.transpose(0, 1).contiguous().transpose(0, 1)      # heads outermost
    assert torch.equal(tkv.qk_norm_rope(by_head, k, pos, f, norm=True, q_weight=qw)[0], want[0])
    got = tkv.qk_norm_rope(q, k, pos, f, v=v, norm=True, q_weight=qw, k_weight=kw, q_out=q, k_out=k, v_out=v)
    assert got[0] is q and all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("t,hq,hkv", [(1501, 32, 4), (6100, 3, 1), (2000, 40, 8)])
def test_long_outputs_over_their_inputs(t, hq, hkv):
    """Enough rows for waves of two octets, also with an odd number of them."""
    q, k, v, qw, kw = _inputs(t, hq, hkv, torch.bfloat16, seed=t, fused=False)
    pos, f = torch.arange(t, device="cuda", dtype=torch.int32), _freq(64)
    want = tkv.qk_norm_rope(q, k, pos, f, v=v, norm=True, q_weight=qw, k_weight=kw)
    some = [0, t // 2, t - 1]
    _check(want[0][some], q[some], pos[some], f, torch.bfloat16, norm=True, weight=qw.double().cpu().numpy())
    _check(want[1][some], k[some], pos[some], f, torch.bfloat16, norm=True, weight=kw.double().cpu().numpy())
    short = tkv.qk_norm_rope(q[-40:], k[-40:], pos[-40:], f, v=v[-40:], norm=True, q_weight=qw, k_weight=kw)
    assert all(torch.equal(a[-40:], b) for a, b in zip(want, short))
    got = tkv.qk_norm_rope(q, k, pos, f, v=v, norm=True, q_weight=qw, k_weight=kw, q_out=q, k_out=k, v_out=v)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_no_tokens():
    q, k, v, _, _ = _inputs(0, 32, 8, torch.float16)
    out = tkv.qk_norm_rope(q, k, torch.zeros(0, dtype=torch.int32, device="cuda"), _freq(128), v=v)
    assert [tuple(x.shape) for x in out] == [(0, 32, 128), (0, 8, 128), (0, 8, 128)]


def test_side_stream_and_replayed_graph():
    q, k, v, qw, kw = _inputs(33, 32, 8, torch.bfloat16)
    pos, f = torch.arange(33, device="cuda", dtype=torch.int32), _freq(128)
    a = dict(v=v, norm=True, q_weight=qw, k_weight=kw, out_dtype=torch.float16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        outs = tkv.qk_norm_rope(q, k, pos, f, **a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        caught = tkv.qk_norm_rope(q, k, pos, f, **a)
    for step in range(4):                    # the positions and rows move on, the graph follows
        graph.replay()
        torch.cuda.synchronize()
        want = tkv.qk_norm_rope(q, k, pos, f, **a)
        assert all(torch.equal(x, y) for x, y in zip(caught, want))
        if step == 0:
            assert all(torch.equal(x, y) for x, y in zip(outs, want))
        pos += 1
        q *= 0.5
