"""PromptAttention used by several threads: what a call hands to the library is its own.  (The library is a stand-in that notes what
it is given.)"""
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
