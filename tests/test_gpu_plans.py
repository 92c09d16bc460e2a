"""PromptAttention and SharedPrefix used by several threads, on several streams and in several graphs: what a call hands to the
library is its own.  (The library is a stand-in that notes what it is given, where nothing else says so.)"""
import ctypes as C
import threading

import pytest
import torch

import paper_2505_19586_amd as tkv
from paper_2505_19586_amd import tkv as binding

pytestmark = pytest.mark.gpu
SM = 128 ** -0.5


class _Notes:
    """Stands for the library: `during` is called with the arguments of every entry."""

    def __init__(self, during):
        self._during = during

    def __getattr__(self, name):
        return lambda *args: self._during(name, args) or 0


def _rows(n, heads, gen, batch=None):
    shape = (n, heads, 128) if batch is None else (batch, n, heads, 128)
    return torch.randn(*shape, generator=gen, device="cuda").half()


def test_a_call_reads_its_own_strides(monkeypatch):
    """A second call with other strides, made while the first is in the library (another thread's, the interpreter's lock is free there)."""
    print("case strides of two calls", flush=True)
    plan = tkv.PromptAttention(n_q_heads=8, n_kv_heads=2)
    g = torch.Generator(device="cuda").manual_seed(0)
    narrow = [_rows(6, h, g) for h in (8, 2, 2)]
    wide = _rows(6, 12, g)
    wide = [wide[:, :8], wide[:, 8:10], wide[:, 10:]]
    seen = []

    def during(name, args):
        if not seen:
            seen.append(None)
            other = threading.Thread(target=plan.attend, args=(*wide, SM, [6]))
            other.start()
            other.join(0.5)  # (it may have to wait until this call has ended)
            seen[0] = list(args[0]._obj.strides)
            waits.append(other)

    waits = []
    monkeypatch.setattr(binding, "lib", lambda: _Notes(during))
    plan.attend(*narrow, SM, [6])
    waits[0].join()
    assert seen[0] == [1024, 128, 256, 128, 256, 128, 1024, 128]


def _workspaces_of(monkeypatch, call, entry, at):
    """Addresses of the workspaces that `call` hands over, in order."""
    got = []
    monkeypatch.setattr(binding, "lib", lambda: _Notes(lambda name, args: got.append(args[at]) if name == entry else None))
    call()
    monkeypatch.undo()
    return got


def _prompt_call(gen):
    plan = tkv.PromptAttention(n_q_heads=8, n_kv_heads=2)
    q, k, v = _rows(3, 8, gen), _rows(3000, 2, gen), _rows(3000, 2, gen)
    return plan, (lambda **kw: plan.attend(q, k, v, SM, [3], [3000], **kw)), "tkv_prompt_attn", 11


def _shared_call(gen):
    P, L = (tkv.QuantLayer(n_q_heads=8, n_kv_heads=2, capacity=4096, batch=b) for b in (1, 3))
    P.append(_rows(3000, 2, gen, 1), _rows(3000, 2, gen, 1))
    L.append(_rows(70, 2, gen, 3), _rows(70, 2, gen, 3))
    plan, q = tkv.SharedPrefix(P, L), _rows(3, 8, gen)
    return plan, (lambda **kw: plan.attn_decode(q, SM, **kw)), "tkv_quant_attn_decode_shared", 8


@pytest.mark.filterwarnings("ignore:The CUDA Graph is empty")  # (the stand-in launches nothing)
@pytest.mark.parametrize("make", [_prompt_call, _shared_call])
def test_streams_and_graphs_have_workspaces_of_their_own(make, monkeypatch):
    print(f"case workspaces {make.__name__}", flush=True)
    plan, call, entry, at = make(torch.Generator(device="cuda").manual_seed(1))
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()

    def on(stream):
        with torch.cuda.stream(stream):
            call()

    def calls():
        call()
        call()
        on(a)
        call(stream=b)
        call(stream=a)
        call(stream=b.cuda_stream)

    w = _workspaces_of(monkeypatch, calls, entry, at)
    assert w[0] == w[1] == plan.workspace.data_ptr()           # a stream's calls follow each other: they share one
    assert w[2] == w[4] and w[3] == w[5] and len({w[0], w[2], w[3]}) == 3
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    outs = []

    def capture():
        for g in graphs:
            with torch.cuda.graph(g):
                outs.append(call())

    captured = _workspaces_of(monkeypatch, capture, entry, at)
    assert len(set(captured) | {w[0], w[2], w[3]}) == 5         # two graphs may be replayed beside each other


@pytest.mark.parametrize("make", [_prompt_call, _shared_call])
def test_graphs_streams_and_threads_at_once(make):
    """Two captured graphs replayed on two streams, eager calls on a third and from two threads: the outputs of one call alone."""
    print(f"case at once {make.__name__}", flush=True)
    _, call, _, _ = make(torch.Generator(device="cuda").manual_seed(2))
    want = call()
    torch.cuda.synchronize()
    graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for g in graphs:
        with torch.cuda.graph(g):
            outs.append(call())
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    eager = []
    for _ in range(8):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        eager.append(call(stream=streams[2]))
        eager.append(call())
    torch.cuda.synchronize()
    assert all(torch.equal(want, o) for o in outs + eager)
    found = [[], []]

    def many(into):
        for _ in range(50):
            into.append(call())

    threads = [threading.Thread(target=many, args=(x,)) for x in found]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert all(torch.equal(want, o) for x in found for o in x) and len(found[0]) == len(found[1]) == 50
