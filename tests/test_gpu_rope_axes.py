"""tkv_qk_norm_rope_axes against float64 and against the one-axis entry point.  Tolerance as in test_gpu_rope: half a step of the
output's type and 2^-19 of |a| + |b| of the channel's pair for float32's errors."""
import numpy as np
import pytest
import torch

import paper_2505_19586_amd as tkv
from oracle.rope import norm_rope
from test_gpu_rope import F32, _freq, _inputs

pytestmark = pytest.mark.gpu


def _check(got, x, pos, axis_of, freq, dtype, **kw):
    at = pos.cpu().numpy()[list(axis_of)].T          # [T, R / 2]
    ref, size = norm_rope(x.double().cpu().numpy(), at, freq.cpu().numpy(), **kw)
    tiny = 2.0 ** -25 if dtype == torch.float16 else 0.0
    assert (np.abs(got.double().cpu().numpy() - ref) <= torch.finfo(dtype).eps / 2 * np.abs(ref) + F32 * size + tiny).all()


def _positions(axes, t, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-1000, 131072, (axes, t), generator=g, device="cuda", dtype=torch.int32)


@pytest.mark.parametrize("src,dst", [(torch.float16, torch.float16), (torch.bfloat16, torch.float16), (torch.bfloat16, torch.bfloat16)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("sections,mixed", [((16, 24, 24), False), ((22, 21, 21), True), ((64,), False), ((0, 64), False), ((10, 20, 4, 30), True),
                                            ((8, 12, 12), False), ((4, 4), True)])
def test_sections(src, dst, interleaved, sections, mixed):
    t = 37
    q, k, v, qw, kw = _inputs(t, 5, 1, src)
    axis_of, pos = tkv.rope_axes(sections, mixed), _positions(len(sections), t)
    f = _freq(2 * sum(sections))
    oq, ok, ov = tkv.qk_norm_rope(q, k, pos, f, v=v, axis_of=axis_of, norm=True, q_weight=qw, k_weight=kw, interleaved=interleaved, out_dtype=dst)
    for o, x, w in ((oq, q, qw), (ok, k, kw)):
        _check(o, x, pos, axis_of, f, dst, norm=True, weight=w.double().cpu().numpy(), interleaved=interleaved)
    assert torch.equal(ov, v.to(dst))


@pytest.mark.parametrize("t", [1, 3, 64, 5001])
def test_axes_that_agree_give_the_bits_of_one(t):
    q, k, v, qw, kw = _inputs(t, 32, 8, torch.bfloat16, seed=t)
    pos, f = _positions(1, t, t), _freq(128)
    a = dict(v=v, norm=True, q_weight=qw, k_weight=kw)
    want = tkv.qk_norm_rope(q, k, pos[0], f, **a)
    for axis_of, p in ((tkv.rope_axes((20, 22, 22)), pos.expand(3, t).contiguous()), (bytes(64), pos),
                       ([2] * 64, torch.cat((_positions(2, t, 5), pos)))):
        assert all(torch.equal(x, y) for x, y in zip(tkv.qk_norm_rope(q, k, p, f, axis_of=axis_of, **a), want))


def test_replayed_graph_and_side_stream():
    q, k, v, qw, kw = _inputs(33, 32, 8, torch.float16)
    pos, f, axis_of = _positions(3, 33), _freq(128), tkv.rope_axes((16, 24, 24))
    a = dict(v=v, axis_of=axis_of, norm=True, q_weight=qw, k_weight=kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    outs = tkv.qk_norm_rope(q, k, pos, f, stream=side, **a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        caught = tkv.qk_norm_rope(q, k, pos, f, **a)
    for step in range(4):
        graph.replay()
        torch.cuda.synchronize()
        want = tkv.qk_norm_rope(q, k, pos, f, **a)
        assert all(torch.equal(x, y) for x, y in zip(caught, want))
        if step == 0:
            assert all(torch.equal(x, y) for x, y in zip(outs, want))
        pos += torch.tensor([[1], [0], [3]], device="cuda", dtype=torch.int32)


def test_wrong_numbers_of_axes_are_refused():
    q, k, _, _, _ = _inputs(4, 2, 1, torch.float16)
    f = _freq(128)
    for pos, axis_of in ((_positions(1, 4), bytes([1] * 64)), (_positions(5, 4), bytes(64))):
        with pytest.raises(tkv.TkvError):
            tkv.qk_norm_rope(q, k, pos, f, axis_of=axis_of)
    with pytest.raises(AssertionError):
        tkv.qk_norm_rope(q, k, _positions(2, 4), f, axis_of=bytes(63))
