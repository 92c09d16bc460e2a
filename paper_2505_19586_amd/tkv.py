"""ctypes binding of libtkv.so: same entry points as include/tkv.h, argument
marshalling only.  Every step of the path runs in the library's HIP kernels; there
is no CPU or PyTorch fallback - a missing library or GPU raises."""
from __future__ import annotations

import ctypes as C
import itertools
import operator
import os
import struct
import threading

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = None

TKV_MAX_BATCH = 64


class TkvError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().tkv_strerror(status).decode() if _LIB is not None else "?"
        super().__init__(f"{where}: {msg} ({status})")


def library_path() -> str:
    return os.path.join(_HERE, "libtkv.so")


class QuantDesc(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("bits", C.c_int32), ("group_size", C.c_int32),
                ("residual", C.c_int32), ("capacity", C.c_int32), ("batch", C.c_int32)]


class QuantCache(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("k_codes", "k_scale", "k_zero", "v_codes", "v_scale", "v_zero",
                                          "k_resid", "v_resid")] + [("seq_len_host", C.POINTER(C.c_int32))]


class SparseDesc(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("n_channels", C.c_int32), ("top_k", C.c_int32),
                ("n_sink", C.c_int32), ("n_window", C.c_int32), ("capacity", C.c_int32), ("batch", C.c_int32)]


class SparseCache(C.Structure):
    _fields_ = [("key_summary", C.c_void_p), ("channel_idx", C.c_void_p), ("kv_host", C.c_void_p),
                ("kv_local", C.c_void_p), ("seq_len_host", C.POINTER(C.c_int32))]


class PrefDesc(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("n_q", C.c_int32), ("top_k", C.c_int32), ("capacity", C.c_int32),
                ("batch", C.c_int32)]


class SparseStage1(C.Structure):
    _fields_ = [("k_absmax", C.c_void_p), ("keys_cm", C.c_void_p)]


class RopeDesc(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("in_dtype", C.c_int32), ("out_dtype", C.c_int32), ("norm", C.c_int32),
                ("eps", C.c_float), ("rotary_dim", C.c_int32), ("interleaved", C.c_int32),
                # (strides of tokens and heads; single fields, as an array each costs a third of a microsecond to fill)
                ("q_stride", C.c_int64), ("q_stride_head", C.c_int64), ("k_stride", C.c_int64),
                ("k_stride_head", C.c_int64), ("v_stride", C.c_int64), ("v_stride_head", C.c_int64)]


# A RopeDesc's bytes: packed by `struct` in a fifth of the time that the class takes for its seventeen fields.
_ROPE_DESC = struct.Struct("Iiiiiiifiiqqqqqq")
assert _ROPE_DESC.size == C.sizeof(RopeDesc)


class PromptDesc(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("dtype", C.c_int32), ("causal", C.c_int32), ("batch", C.c_int32),
                ("reserved", C.c_int32), ("strides", C.c_int64 * 8)]  # of tokens and heads: q, k, v, out


class PagedDesc(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("dtype", C.c_int32), ("bits", C.c_int32), ("page_size", C.c_int32),
                ("n_pages", C.c_int32), ("k_stride", C.c_int64 * 3), ("v_stride", C.c_int64 * 3)]  # of pages, heads, tokens


def lib() -> C.CDLL:
    """Loads libtkv.so (built by paper_2505_19586_amd/build.py); raises if absent."""
    global _LIB
    if _LIB is None:
        path = library_path()
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is missing: build it with `python -m paper_2505_19586_amd.build`")
        L = C.CDLL(path)
        L.tkv_strerror.restype = C.c_char_p
        L.tkv_strerror.argtypes = [C.c_int32]
        vp, i32, sz = C.c_void_p, C.c_int32, C.c_size_t
        L.tkv_quant_cache_sizes.argtypes = [C.POINTER(QuantDesc), C.POINTER(sz), C.POINTER(sz)]
        L.tkv_quantize_append.argtypes = [C.POINTER(QuantDesc), C.POINTER(QuantCache), vp, vp, i32, vp]
        L.tkv_quantize_append_ragged.argtypes = [C.POINTER(QuantDesc), C.POINTER(QuantCache), vp, vp, i32,
                                                 C.POINTER(i32), vp]
        L.tkv_sparse_append_ragged.argtypes = [C.POINTER(SparseDesc), C.POINTER(SparseCache), vp, vp, i32,
                                               C.POINTER(i32), vp]
        L.tkv_quant_attn_decode.argtypes = [C.POINTER(QuantDesc), C.POINTER(QuantCache), vp, vp, C.c_float, vp, sz, vp]
        L.tkv_quant_decode.argtypes = [C.POINTER(QuantDesc), C.POINTER(QuantCache), vp, vp, i32, C.POINTER(i32), vp, vp,
                                       C.c_float, vp, sz, vp]
        L.tkv_quant_attn_decode_static.argtypes = [C.POINTER(QuantDesc), C.POINTER(QuantCache), vp, vp, C.c_float, vp]
        L.tkv_sparse_cache_sizes.argtypes = [C.POINTER(SparseDesc), C.POINTER(sz), C.POINTER(sz)]
        L.tkv_sparse_append.argtypes = [C.POINTER(SparseDesc), C.POINTER(SparseCache), vp, vp, i32, vp]
        L.tkv_sparse_estimate_topk.argtypes = [C.POINTER(SparseDesc), C.POINTER(SparseCache), vp, vp, vp, vp, sz, vp]
        L.tkv_sparse_gather_attn.argtypes = [C.POINTER(SparseDesc), C.POINTER(SparseCache), vp, vp, vp, vp,
                                             C.c_float, vp, vp, sz, vp, vp]
        L.tkv_sparse_gather.argtypes = [C.POINTER(SparseDesc), C.POINTER(SparseCache), vp, vp, vp, vp]
        L.tkv_sparse_attn.argtypes = [C.POINTER(SparseDesc), C.POINTER(SparseCache), vp, vp, vp, vp, C.c_float,
                                      vp, sz, vp]
        L.tkv_sparse_stage1_sizes.argtypes = [C.POINTER(SparseDesc), C.POINTER(sz)]
        L.tkv_sparse_stage1_append.argtypes = [C.POINTER(SparseDesc), C.POINTER(SparseCache), C.POINTER(SparseStage1),
                                               vp, i32, C.POINTER(i32), vp]
        L.tkv_sparse_select_channels.argtypes = [C.POINTER(SparseDesc), C.POINTER(SparseStage1), vp, vp, vp]
        L.tkv_sparse_prefetch_keys.argtypes = [C.POINTER(SparseDesc), C.POINTER(SparseCache), C.POINTER(SparseStage1),
                                               vp, vp, vp]
        L.tkv_sparse_estimate_topk_cm.argtypes = [C.POINTER(SparseDesc), C.POINTER(SparseCache), vp, vp, vp, i32,
                                                  vp, vp, vp, sz, vp]
        L.tkv_sparse_select_estimate_topk.argtypes = [C.POINTER(SparseDesc), C.POINTER(SparseCache),
                                                      C.POINTER(SparseStage1), vp, vp, vp, vp, vp, vp, sz, vp]
        L.tkv_sparse_append_dynamic.argtypes = [C.POINTER(SparseDesc), C.POINTER(SparseCache), C.POINTER(SparseStage1),
                                                vp, vp, i32, C.POINTER(i32), vp]
        L.tkv_sparse_decode.argtypes = [C.POINTER(SparseDesc), C.POINTER(SparseCache), vp, vp, i32, C.POINTER(i32),
                                        vp, vp, vp, vp, C.c_float, vp, vp, sz, vp]
        L.tkv_sparse_append_estimate_topk.argtypes = [C.POINTER(SparseDesc), C.POINTER(SparseCache), vp, vp, i32,
                                                      C.POINTER(i32), vp, vp, vp, vp, sz, vp]
        L.tkv_dense_preference_sizes.argtypes = [C.POINTER(PrefDesc), C.POINTER(sz)]
        L.tkv_dense_preference.argtypes = [C.POINTER(PrefDesc), vp, vp, i32, C.c_float, vp, vp, sz, vp]
        L.tkv_classify_layer.argtypes = [C.POINTER(C.c_float), i32, i32, C.c_float, C.POINTER(C.c_float)]
        L.tkv_qk_norm_rope.argtypes = [vp, i32] + [vp] * 11  # (a descriptor's bytes or its reference)
        L.tkv_qk_norm_rope_axes.argtypes = [vp, i32] + [vp] * 6 + [i32] + [vp] * 6
        L.tkv_paged_cache_sizes.argtypes = [C.POINTER(PagedDesc), C.POINTER(sz)]
        L.tkv_paged_append.argtypes = [vp, vp, i32] + [vp] * 6 + [i32] + [vp] * 8
        L.tkv_paged_gather.argtypes = [vp, vp, vp, i32] + [vp] * 4
        L.tkv_paged_attn_sizes.argtypes = [C.POINTER(PagedDesc), C.POINTER(sz)]
        L.tkv_paged_attn.argtypes = [vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, i32, vp, vp, i32, C.c_float, vp, sz, vp]
        L.tkv_prompt_attn_sizes.argtypes = [C.POINTER(PromptDesc), C.POINTER(sz)]
        L.tkv_prompt_attn.argtypes = [C.POINTER(PromptDesc)] + [vp] * 9 + [C.c_float, vp, sz, vp]
        L.tkv_quant_attn_decode_shared_sizes.argtypes = [C.POINTER(QuantDesc), C.POINTER(QuantDesc), C.POINTER(sz)]
        L.tkv_quant_attn_decode_shared.argtypes = [C.POINTER(QuantDesc), C.POINTER(QuantCache), C.POINTER(QuantDesc),
                                                   C.POINTER(QuantCache), vp, vp, vp, C.c_float, vp, sz, vp]
        L.tkv_debug_quant_attn_config.argtypes = [i32, i32]
        L.tkv_debug_quant_attn_config.restype = i32
        L.tkv_debug_read_sweep.argtypes = [vp, C.c_size_t, vp, i32, vp]
        L.tkv_debug_read_sweep.restype = i32
        for name in ("tkv_quant_cache_sizes", "tkv_quantize_append", "tkv_quant_attn_decode",
                     "tkv_quant_attn_decode_static",
                     "tkv_quantize_append_ragged", "tkv_sparse_append_ragged",
                     "tkv_sparse_cache_sizes", "tkv_sparse_append", "tkv_sparse_estimate_topk",
                     "tkv_sparse_gather_attn", "tkv_sparse_gather", "tkv_sparse_attn",
                     "tkv_sparse_stage1_sizes", "tkv_sparse_stage1_append", "tkv_sparse_select_channels",
                     "tkv_sparse_prefetch_keys", "tkv_sparse_estimate_topk_cm",
                     "tkv_sparse_select_estimate_topk", "tkv_sparse_append_dynamic",
                     "tkv_sparse_append_estimate_topk", "tkv_sparse_decode", "tkv_dense_preference_sizes", "tkv_dense_preference",
                     "tkv_classify_layer", "tkv_qk_norm_rope", "tkv_qk_norm_rope_axes", "tkv_paged_cache_sizes",
                     "tkv_paged_append", "tkv_paged_gather", "tkv_paged_attn_sizes", "tkv_paged_attn",
                     "tkv_prompt_attn_sizes", "tkv_prompt_attn", "tkv_quant_attn_decode_shared_sizes",
                     "tkv_quant_attn_decode_shared"):
            getattr(L, name).restype = C.c_int32
        _LIB = L
    return _LIB


def debug_quant_attn_config(kernel_choice: int = 0, target_blocks: int = 0) -> None:
    """0 = the setting's own kernel (default), 1 = reference kernel; see tkv_debug.h."""
    _check(lib().tkv_debug_quant_attn_config(int(kernel_choice), int(target_blocks)), "tkv_debug_quant_attn_config")


def debug_read_sweep(buf: torch.Tensor, n_workgroups: int = 2048, stream=None) -> None:
    """Measurement aid: one plain read sweep over a device tensor (size a multiple of 16 bytes)."""
    assert buf.is_cuda and buf.is_contiguous()
    _check(lib().tkv_debug_read_sweep(buf.data_ptr(), buf.numel() * buf.element_size(), None, int(n_workgroups),
                                      _stream(stream)), "tkv_debug_read_sweep")


def _check(status: int, where: str) -> None:
    if status != 0:
        raise TkvError(status, where)


def _stream(stream) -> int:
    if stream is None:  # the current device's current stream; as an object it costs 2.8 us, a quarter of a short step's call
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _handle(at: int, stream) -> int:
    """_on_current and _stream in one, for tensors of device number `at`."""
    assert at >= 0, "tensors of a GPU"
    if stream is not None:
        return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    current = torch._C._cuda_getDevice()
    assert at == current, f"tensors on device {at}, the current device is {current}: make it current or pass a stream of theirs"
    return torch._C._cuda_getCurrentRawStream(current)


def _on_current(t: torch.Tensor, stream) -> None:
    """Without a stream the current device's is used: the tensors have to be that device's."""
    assert stream is not None or t.get_device() == torch._C._cuda_getDevice(), \
        f"tensors on {t.device}, the current device is another: make it current or pass a stream of theirs"


def _new(shape, dtype, device, stream, fill=None) -> torch.Tensor:
    """A new output, made (and filled) in the order of the stream that will write it."""
    if stream is not None:
        with torch.cuda.stream(stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream), device=device)):
            return _new(shape, dtype, device, None, fill)
    return torch.empty(shape, dtype=dtype, device=device) if fill is None else torch.full(shape, fill, dtype=dtype, device=device)


def _like(x: torch.Tensor, dtype, stream) -> torch.Tensor:
    """A new contiguous output of x's shape.  (empty_like spares a microsecond of torch.empty's two.)"""
    if stream is not None:
        return _new(x.shape, dtype, x.device, stream)
    return torch.empty_like(x, dtype=dtype, memory_format=torch.contiguous_format)


def _given(out: torch.Tensor | None, x: torch.Tensor, dtype, at: int, stream) -> torch.Tensor:
    """An output of x's shape, where the caller gave none a new one."""
    if out is None:
        return _like(x, dtype, stream)
    assert out.dtype == dtype and out.shape == x.shape and out.is_contiguous() and out.get_device() == at
    return out


class _Workspaces:
    """The workspaces of an object's calls: one for every stream, whose calls follow each other, and one of its own for every call made
    while the current stream is captured into a graph (it stays in the graph's memory pool), as graphs may be replayed beside each
    other and beside eager calls.  Threads hold `lock` while their call's launches go out, so that none of another thread's, with
    the same workspace, comes in between."""

    def __init__(self, n_bytes: int, device: torch.device, at_once: bool = True, zeros: int = 0):
        """zeros: bytes at the end that are zero-filled when a workspace is made."""
        self._bytes, self._device, self._of, self._zeros = n_bytes, device, {}, zeros
        self.lock = threading.Lock()
        if at_once:
            with torch.cuda.device(device):
                self.of(_stream(None))

    def of(self, handle: int, stream=None) -> torch.Tensor:
        captured = torch._C._cuda_isCurrentStreamCapturing()
        w = None if captured else self._of.get(handle)
        if w is None:
            w = _new(self._bytes, torch.uint8, self._device, stream)
            if self._zeros and stream is None:
                w[-self._zeros:].zero_()
            elif self._zeros:
                with torch.cuda.stream(stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(handle, device=self._device)):
                    w[-self._zeros:].zero_()
            if not captured:
                self._of[handle] = w
        return w


def _ptr(t) -> int:
    return 0 if t is None else t.data_ptr()


def _require_gpu(device) -> torch.device:
    if not torch.cuda.is_available():
        raise RuntimeError("tkv needs an AMD GPU (gfx950); no CPU fallback exists")
    return torch.device(device)


class QuantLayer:
    """Buffers of one quantization-friendly layer plus the three entry points that
    act on them (tkv_quant_cache_sizes, tkv_quantize_append, tkv_quant_attn_decode)."""

    def __init__(self, *, n_q_heads=32, n_kv_heads=8, head_dim=128, bits=2, group_size=32, residual=128,
                 capacity, batch=1, device="cuda:0"):
        dev = _require_gpu(device)
        self.desc = QuantDesc(C.sizeof(QuantDesc), n_q_heads, n_kv_heads, head_dim, bits, group_size, residual,
                              capacity, batch)
        sizes = (C.c_size_t * 8)()
        ws = C.c_size_t()
        _check(lib().tkv_quant_cache_sizes(C.byref(self.desc), sizes, C.byref(ws)), "tkv_quant_cache_sizes")
        self.sizes = [int(s) for s in sizes]
        self.workspace_bytes = int(ws.value)
        names = ("k_codes", "k_scale", "k_zero", "v_codes", "v_scale", "v_zero", "k_resid", "v_resid")
        self.buffers = {n: torch.zeros(max(s, 16), dtype=torch.uint8, device=dev) for n, s in zip(names, self.sizes)}
        # zero once: the arrival counters behind the partials must start at zero
        self.workspace = torch.zeros(self.workspace_bytes, dtype=torch.uint8, device=dev)
        self.seq_len = np.zeros(batch, dtype=np.int32)
        self.cache = QuantCache(*[self.buffers[n].data_ptr() for n in names],
                                self.seq_len.ctypes.data_as(C.POINTER(C.c_int32)))
        self.device = dev

    def append(self, k_new: torch.Tensor, v_new: torch.Tensor, n_valid=None, stream=None) -> None:
        """k_new, v_new: fp16 [B, n_new, Hkv, D] on the device; n_valid: optional
        per-sequence row counts (padded batch)."""
        d = self.desc
        assert k_new.dtype == torch.float16 and v_new.dtype == torch.float16
        assert k_new.is_cuda and k_new.is_contiguous() and v_new.is_contiguous()
        assert tuple(k_new.shape) == tuple(v_new.shape) and k_new.shape[0] == d.batch
        assert tuple(k_new.shape[2:]) == (d.n_kv_heads, d.head_dim)
        if n_valid is None:
            _check(lib().tkv_quantize_append(C.byref(d), C.byref(self.cache), k_new.data_ptr(), v_new.data_ptr(),
                                             int(k_new.shape[1]), _stream(stream)), "tkv_quantize_append")
        else:
            nv = np.ascontiguousarray(n_valid, dtype=np.int32)
            assert nv.shape == (d.batch,)
            _check(lib().tkv_quantize_append_ragged(C.byref(d), C.byref(self.cache), k_new.data_ptr(),
                                                    v_new.data_ptr(), int(k_new.shape[1]),
                                                    nv.ctypes.data_as(C.POINTER(C.c_int32)), _stream(stream)),
                   "tkv_quantize_append_ragged")

    def attn_decode(self, q: torch.Tensor, sm_scale: float, out: torch.Tensor | None = None, stream=None):
        d = self.desc
        assert q.dtype == torch.float16 and q.is_cuda and q.is_contiguous()
        assert tuple(q.shape) == (d.batch, d.n_q_heads, d.head_dim)
        if out is None:
            out = torch.empty_like(q)
        _check(lib().tkv_quant_attn_decode(C.byref(d), C.byref(self.cache), q.data_ptr(), out.data_ptr(),
                                           float(sm_scale), self.workspace.data_ptr(), self.workspace_bytes,
                                           _stream(stream)), "tkv_quant_attn_decode")
        return out

    def decode(self, q: torch.Tensor, sm_scale: float, k_new: torch.Tensor, v_new: torch.Tensor, n_valid=None,
               out: torch.Tensor | None = None, stream=None):
        """tkv_quant_decode: the step's append and the attention over the grown cache in one call
        (no launch for the append, but for few steps; see tkv_quant_decode)."""
        d = self.desc
        assert q.dtype == torch.float16 and q.is_cuda and q.is_contiguous()
        assert tuple(q.shape) == (d.batch, d.n_q_heads, d.head_dim)
        assert k_new.dtype == torch.float16 and v_new.dtype == torch.float16
        assert k_new.is_cuda and k_new.is_contiguous() and v_new.is_contiguous()
        assert tuple(k_new.shape) == tuple(v_new.shape) and k_new.shape[0] == d.batch
        assert tuple(k_new.shape[2:]) == (d.n_kv_heads, d.head_dim)
        nv = None
        if n_valid is not None:
            nv = np.ascontiguousarray(n_valid, dtype=np.int32)
            assert nv.shape == (d.batch,)
        if out is None:
            out = torch.empty_like(q)
        _check(lib().tkv_quant_decode(C.byref(d), C.byref(self.cache), k_new.data_ptr(), v_new.data_ptr(),
                                      int(k_new.shape[1]),
                                      None if nv is None else nv.ctypes.data_as(C.POINTER(C.c_int32)),
                                      q.data_ptr(), out.data_ptr(), float(sm_scale), self.workspace.data_ptr(),
                                      self.workspace_bytes, _stream(stream)), "tkv_quant_decode")
        return out

    def attn_decode_static(self, q: torch.Tensor, sm_scale: float, out: torch.Tensor, stream=None):
        """tkv_quant_attn_decode_static: no workspace, nothing allocated (the caller passes `out`)."""
        d = self.desc
        assert q.dtype == torch.float16 and q.is_cuda and q.is_contiguous()
        assert out.dtype == torch.float16 and out.is_cuda and out.is_contiguous() and out.shape == q.shape
        assert tuple(q.shape) == (d.batch, d.n_q_heads, d.head_dim)
        _check(lib().tkv_quant_attn_decode_static(C.byref(d), C.byref(self.cache), q.data_ptr(), out.data_ptr(),
                                                  float(sm_scale), _stream(stream)), "tkv_quant_attn_decode_static")
        return out

    # typed views of the raw buffers (for tests)
    def view(self, name: str) -> torch.Tensor:
        d = self.desc
        bh = (d.batch, d.n_kv_heads)
        j = d.capacity // 32   # codes and value scalers / zero-points: blocks of 32 tokens
        buf = self.buffers[name]
        if name in ("k_codes", "v_codes"):
            return buf.view(torch.int32).view(*bh, j, 128 * d.bits)
        if name in ("k_scale", "k_zero"):
            return buf.view(torch.float16).view(*bh, d.capacity // d.group_size, 128)
        if name in ("v_scale", "v_zero"):
            return buf.view(torch.float16).view(*bh, j, 128 // d.group_size, 32)
        return buf.view(torch.float16).view(*bh, d.residual + d.group_size, 128)


class SharedPrefix:
    """Decode attention of a batch (`layer`) whose sequences share prefixes, each held once in `prefix`
    (tkv_quant_attn_decode_shared).  Both are ordinary QuantLayers: append a prompt to `prefix`, every sequence's own
    tokens to `layer`.  Streams, threads and captured graphs may use one object at the same time (each stream and graph has a workspace
    of its own); a graph keeps the numbers of tokens that it was captured with."""

    def __init__(self, prefix: QuantLayer, layer: QuantLayer):
        ws = C.c_size_t()
        _check(lib().tkv_quant_attn_decode_shared_sizes(C.byref(prefix.desc), C.byref(layer.desc), C.byref(ws)),
               "tkv_quant_attn_decode_shared_sizes")
        assert prefix.workspace.device == layer.workspace.device
        self.prefix, self.layer = prefix, layer
        self.workspace_bytes = int(ws.value)
        self._device = layer.workspace.device
        self._workspaces = _Workspaces(self.workspace_bytes, self._device)

    @property
    def workspace(self) -> torch.Tensor:
        """That of the current stream's calls."""
        return self._workspaces.of(_stream(None))

    def attn_decode(self, q: torch.Tensor, sm_scale: float, prefix_of=None, out: torch.Tensor | None = None, stream=None):
        """q fp16 [B, Hq, 128]; prefix_of: for every sequence the prefix it continues, -1 for none (default: 0 for all)."""
        d = self.layer.desc
        assert q.dtype == torch.float16 and q.is_contiguous() and tuple(q.shape) == (d.batch, d.n_q_heads, d.head_dim)
        assert q.device == self._device
        _on_current(q, stream)
        of = None
        if prefix_of is not None:
            of = np.ascontiguousarray(prefix_of, dtype=np.int32)
            assert of.shape == (d.batch,)
            of_at = of.__array_interface__["data"][0]
        if out is None:
            out = _new(q.shape, q.dtype, q.device, stream)
        else:
            assert out.dtype == torch.float16 and out.is_contiguous() and out.shape == q.shape and out.device == q.device
        handle = _stream(stream)
        with self._workspaces.lock:
            workspace = self._workspaces.of(handle, stream)
            status = lib().tkv_quant_attn_decode_shared(C.byref(self.prefix.desc), C.byref(self.prefix.cache), C.byref(d),
                                                        C.byref(self.layer.cache), None if of is None else of_at, q.data_ptr(),
                                                        out.data_ptr(), float(sm_scale), workspace.data_ptr(), self.workspace_bytes,
                                                        handle)
        _check(status, "tkv_quant_attn_decode_shared")
        return out


class SparseLayer:
    """Buffers of one sparsity-friendly layer (GPU key summary, pinned host K/V,
    resident sink/window rows) and the entry points that act on them."""

    def __init__(self, *, n_q_heads=32, n_kv_heads=8, head_dim=128, n_channels=16, top_k=1024, n_sink=4,
                 n_window=64, capacity, batch=1, device="cuda:0", kv_host: torch.Tensor | None = None):
        dev = _require_gpu(device)
        self.desc = SparseDesc(C.sizeof(SparseDesc), n_q_heads, n_kv_heads, head_dim, n_channels, top_k, n_sink,
                               n_window, capacity, batch)
        sizes = (C.c_size_t * 4)()
        ws = C.c_size_t()
        _check(lib().tkv_sparse_cache_sizes(C.byref(self.desc), sizes, C.byref(ws)), "tkv_sparse_cache_sizes")
        self.sizes = [int(s) for s in sizes]
        self.workspace_bytes = int(ws.value)
        self.key_summary = torch.zeros(self.sizes[0] // 2, dtype=torch.float16, device=dev).view(
            batch, n_kv_heads, capacity, n_channels)
        self.channel_idx = torch.zeros(batch, n_kv_heads, n_channels, dtype=torch.int32, device=dev)
        if kv_host is None:
            kv_host = torch.empty(self.sizes[2] // 2, dtype=torch.float16, pin_memory=True)
        assert kv_host.is_pinned() and kv_host.numel() * 2 >= self.sizes[2]
        self.kv_host = kv_host.view(-1)[: self.sizes[2] // 2].view(batch, n_kv_heads, capacity, 2, head_dim)
        self.kv_local = torch.zeros(batch, n_kv_heads, n_sink + n_window, 2, head_dim, dtype=torch.float16, device=dev)
        # zero once: the Top-K histogram and counters must start at zero (each call leaves them zero)
        self.workspace = torch.zeros(self.workspace_bytes, dtype=torch.uint8, device=dev)
        self.staging = torch.empty(batch, n_kv_heads, top_k, 2, head_dim, dtype=torch.float16, device=dev)
        self.topk_idx = torch.empty(batch, n_kv_heads, top_k, dtype=torch.int32, device=dev)
        self.topk_count = torch.zeros(batch, n_kv_heads, dtype=torch.int32, device=dev)
        self.seq_len = np.zeros(batch, dtype=np.int32)
        self.cache = SparseCache(self.key_summary.data_ptr(), self.channel_idx.data_ptr(), self.kv_host.data_ptr(),
                                 self.kv_local.data_ptr(), self.seq_len.ctypes.data_as(C.POINTER(C.c_int32)))
        self.device = dev

    def set_channels(self, channel_idx) -> None:
        if not isinstance(channel_idx, torch.Tensor):
            channel_idx = torch.from_numpy(np.ascontiguousarray(channel_idx, dtype=np.int32))
        self.channel_idx.copy_(channel_idx.to(torch.int32).reshape(self.channel_idx.shape))

    def append(self, k_new: torch.Tensor, v_new: torch.Tensor, n_valid=None, stream=None) -> None:
        d = self.desc
        assert k_new.dtype == torch.float16 and k_new.is_cuda and k_new.is_contiguous() and v_new.is_contiguous()
        assert tuple(k_new.shape) == tuple(v_new.shape) and k_new.shape[0] == d.batch
        assert tuple(k_new.shape[2:]) == (d.n_kv_heads, d.head_dim)
        if n_valid is None:
            _check(lib().tkv_sparse_append(C.byref(d), C.byref(self.cache), k_new.data_ptr(), v_new.data_ptr(),
                                           int(k_new.shape[1]), _stream(stream)), "tkv_sparse_append")
        else:
            nv = np.ascontiguousarray(n_valid, dtype=np.int32)
            assert nv.shape == (d.batch,)
            _check(lib().tkv_sparse_append_ragged(C.byref(d), C.byref(self.cache), k_new.data_ptr(),
                                                  v_new.data_ptr(), int(k_new.shape[1]),
                                                  nv.ctypes.data_as(C.POINTER(C.c_int32)), _stream(stream)),
                   "tkv_sparse_append_ragged")

    def estimate_topk(self, q: torch.Tensor, stream=None):
        d = self.desc
        assert q.dtype == torch.float16 and q.is_cuda and q.is_contiguous()
        assert tuple(q.shape) == (d.batch, d.n_q_heads, d.head_dim)
        _check(lib().tkv_sparse_estimate_topk(C.byref(d), C.byref(self.cache), q.data_ptr(),
                                              self.topk_idx.data_ptr(), self.topk_count.data_ptr(),
                                              self.workspace.data_ptr(), self.workspace_bytes, _stream(stream)),
               "tkv_sparse_estimate_topk")
        return self.topk_idx, self.topk_count

    def append_estimate_topk(self, k_new: torch.Tensor, v_new: torch.Tensor, q: torch.Tensor, n_valid=None,
                             stream=None):
        """A decode step's append and estimate_topk in one call (at most 8 new tokens)."""
        d = self.desc
        assert k_new.dtype == torch.float16 and k_new.is_cuda and k_new.is_contiguous() and v_new.is_contiguous()
        assert tuple(k_new.shape) == tuple(v_new.shape) and k_new.shape[0] == d.batch
        assert tuple(k_new.shape[2:]) == (d.n_kv_heads, d.head_dim)
        assert q.dtype == torch.float16 and q.is_cuda and q.is_contiguous()
        assert tuple(q.shape) == (d.batch, d.n_q_heads, d.head_dim)
        nv = None
        if n_valid is not None:
            nv = np.ascontiguousarray(n_valid, dtype=np.int32)
            assert nv.shape == (d.batch,)
        _check(lib().tkv_sparse_append_estimate_topk(
            C.byref(d), C.byref(self.cache), k_new.data_ptr(), v_new.data_ptr(), int(k_new.shape[1]),
            None if nv is None else nv.ctypes.data_as(C.POINTER(C.c_int32)), q.data_ptr(),
            self.topk_idx.data_ptr(), self.topk_count.data_ptr(), self.workspace.data_ptr(), self.workspace_bytes,
            _stream(stream)), "tkv_sparse_append_estimate_topk")
        return self.topk_idx, self.topk_count

    def decode(self, q: torch.Tensor, sm_scale: float, k_new: torch.Tensor | None = None,
               v_new: torch.Tensor | None = None, n_valid=None, out: torch.Tensor | None = None, stream=None,
               warm_next: "SparseLayer | None" = None):
        """tkv_sparse_decode: the step's append (if k_new is given), scoring, Top-K, fetch of the
        selected rows and attention in one launch.  warm_next: the sparse layer (same shape) whose
        decode is the stream's next call: its key summary is read once while this call waits for
        the host link."""
        d = self.desc
        assert q.dtype == torch.float16 and q.is_cuda and q.is_contiguous()
        assert tuple(q.shape) == (d.batch, d.n_q_heads, d.head_dim)
        n_new, kp, vp_, nv = 0, None, None, None
        if k_new is not None:
            assert k_new.dtype == torch.float16 and k_new.is_cuda and k_new.is_contiguous() and v_new.is_contiguous()
            assert tuple(k_new.shape) == tuple(v_new.shape) and k_new.shape[0] == d.batch
            assert tuple(k_new.shape[2:]) == (d.n_kv_heads, d.head_dim)
            n_new, kp, vp_ = int(k_new.shape[1]), k_new.data_ptr(), v_new.data_ptr()
            if n_valid is not None:
                nv = np.ascontiguousarray(n_valid, dtype=np.int32)
                assert nv.shape == (d.batch,)
        if out is None:
            out = torch.empty_like(q)
        warm_ptr = None
        if warm_next is not None:
            assert bytes(warm_next.desc) == bytes(d), "warm_next must have this layer's descriptor"
            warm_ptr = warm_next.key_summary.data_ptr()
        _check(lib().tkv_sparse_decode(
            C.byref(d), C.byref(self.cache), kp, vp_, n_new,
            None if nv is None else nv.ctypes.data_as(C.POINTER(C.c_int32)), q.data_ptr(),
            self.topk_idx.data_ptr(), self.topk_count.data_ptr(), out.data_ptr(), float(sm_scale),
            warm_ptr, self.workspace.data_ptr(), self.workspace_bytes, _stream(stream)),
            "tkv_sparse_decode")
        return out

    def gather_attn(self, q: torch.Tensor, sm_scale: float, out: torch.Tensor | None = None,
                    gather_stream=None, compute_stream=None):
        d = self.desc
        assert q.dtype == torch.float16 and q.is_cuda and q.is_contiguous()
        if out is None:
            out = torch.empty_like(q)
        cs = _stream(compute_stream)
        gs = cs if gather_stream is None else _stream(gather_stream)
        _check(lib().tkv_sparse_gather_attn(C.byref(d), C.byref(self.cache), q.data_ptr(), self.topk_idx.data_ptr(),
                                            self.topk_count.data_ptr(), out.data_ptr(), float(sm_scale),
                                            self.staging.data_ptr(), self.workspace.data_ptr(),
                                            self.workspace_bytes, gs, cs), "tkv_sparse_gather_attn")
        return out

    def gather(self, stream=None) -> None:
        _check(lib().tkv_sparse_gather(C.byref(self.desc), C.byref(self.cache), self.topk_idx.data_ptr(),
                                       self.topk_count.data_ptr(), self.staging.data_ptr(), _stream(stream)),
               "tkv_sparse_gather")

    def attn(self, q: torch.Tensor, sm_scale: float, out: torch.Tensor | None = None, stream=None):
        if out is None:
            out = torch.empty_like(q)
        _check(lib().tkv_sparse_attn(C.byref(self.desc), C.byref(self.cache), q.data_ptr(),
                                     self.topk_count.data_ptr(), self.staging.data_ptr(), out.data_ptr(),
                                     float(sm_scale), self.workspace.data_ptr(), self.workspace_bytes,
                                     _stream(stream)), "tkv_sparse_attn")
        return out


class Stage1:
    """Stage 1 buffers of one sparsity-friendly layer (tkv_sparse_stage1): running
    channel maxima, a channel-major copy of the keys (pinned host memory, or device
    memory with resident=True) and two buffers for the fetched critical key cache."""

    def __init__(self, layer: SparseLayer, resident: bool = False, keys_cm: torch.Tensor | None = None,
                 fetched: list | None = None):
        self.layer = layer
        d = layer.desc
        sizes = (C.c_size_t * 2)()
        _check(lib().tkv_sparse_stage1_sizes(C.byref(d), sizes), "tkv_sparse_stage1_sizes")
        self.k_absmax = torch.zeros(d.batch, d.n_kv_heads, d.head_dim, dtype=torch.float32, device=layer.device)
        if keys_cm is None:
            if resident:
                keys_cm = torch.zeros(int(sizes[1]) // 2, dtype=torch.float16, device=layer.device)
            else:
                keys_cm = torch.zeros(int(sizes[1]) // 2, dtype=torch.float16, pin_memory=True)
        assert keys_cm.numel() * 2 >= int(sizes[1])
        self.resident = keys_cm.is_cuda
        self.keys_cm = keys_cm.view(-1)[: int(sizes[1]) // 2].view(d.batch, d.n_kv_heads, d.head_dim, d.capacity)
        self.channel_idx = torch.zeros(d.batch, d.n_kv_heads, d.n_channels, dtype=torch.int32, device=layer.device)
        if fetched is None:   # double buffer (Sec. 4.2); layers of the same shape may share one pair
            fetched = [torch.zeros(d.batch, d.n_kv_heads, d.n_channels, d.capacity, dtype=torch.float16,
                                   device=layer.device) for _ in range(2)]
        assert len(fetched) == 2 and all(tuple(f.shape) == (d.batch, d.n_kv_heads, d.n_channels, d.capacity)
                                         for f in fetched)
        self.fetched = fetched
        self.s1 = SparseStage1(self.k_absmax.data_ptr(), self.keys_cm.data_ptr())

    def append(self, k_new: torch.Tensor, n_valid=None, stream=None) -> None:
        """Call before layer.append with the same rows."""
        d = self.layer.desc
        assert k_new.dtype == torch.float16 and k_new.is_cuda and k_new.is_contiguous()
        assert k_new.shape[0] == d.batch and tuple(k_new.shape[2:]) == (d.n_kv_heads, d.head_dim)
        nv = None
        if n_valid is not None:
            nv = np.ascontiguousarray(n_valid, dtype=np.int32)
            assert nv.shape == (d.batch,)
        _check(lib().tkv_sparse_stage1_append(C.byref(d), C.byref(self.layer.cache), C.byref(self.s1),
                                              k_new.data_ptr(), int(k_new.shape[1]),
                                              None if nv is None else nv.ctypes.data_as(C.POINTER(C.c_int32)),
                                              _stream(stream)), "tkv_sparse_stage1_append")

    def append_both(self, k_new: torch.Tensor, v_new: torch.Tensor, n_valid=None, stream=None) -> None:
        """Stage 1 buffers and the layer's own cache in one call (tkv_sparse_append_dynamic)."""
        L = self.layer
        d = L.desc
        assert k_new.dtype == torch.float16 and k_new.is_cuda and k_new.is_contiguous() and v_new.is_contiguous()
        assert tuple(k_new.shape) == tuple(v_new.shape) and k_new.shape[0] == d.batch
        assert tuple(k_new.shape[2:]) == (d.n_kv_heads, d.head_dim)
        nv = None
        if n_valid is not None:
            nv = np.ascontiguousarray(n_valid, dtype=np.int32)
            assert nv.shape == (d.batch,)
        _check(lib().tkv_sparse_append_dynamic(C.byref(d), C.byref(L.cache), C.byref(self.s1), k_new.data_ptr(),
                                               v_new.data_ptr(), int(k_new.shape[1]),
                                               None if nv is None else nv.ctypes.data_as(C.POINTER(C.c_int32)),
                                               _stream(stream)), "tkv_sparse_append_dynamic")

    def select_estimate_topk(self, q_hat: torch.Tensor, q: torch.Tensor, stream=None):
        """Eq. 10 and Stage 2 in one call over the resident channel-major keys."""
        L = self.layer
        d = L.desc
        for t in (q_hat, q):
            assert t.dtype == torch.float16 and t.is_cuda and t.is_contiguous()
            assert tuple(t.shape) == (d.batch, d.n_q_heads, d.head_dim)
        _check(lib().tkv_sparse_select_estimate_topk(C.byref(d), C.byref(L.cache), C.byref(self.s1), q_hat.data_ptr(),
                                                     q.data_ptr(), self.channel_idx.data_ptr(), L.topk_idx.data_ptr(),
                                                     L.topk_count.data_ptr(), L.workspace.data_ptr(),
                                                     L.workspace_bytes, _stream(stream)),
               "tkv_sparse_select_estimate_topk")
        return L.topk_idx, L.topk_count

    def select_channels(self, q_hat: torch.Tensor, stream=None) -> torch.Tensor:
        d = self.layer.desc
        assert q_hat.dtype == torch.float16 and q_hat.is_cuda and q_hat.is_contiguous()
        assert tuple(q_hat.shape) == (d.batch, d.n_q_heads, d.head_dim)
        _check(lib().tkv_sparse_select_channels(C.byref(d), C.byref(self.s1), q_hat.data_ptr(),
                                                self.channel_idx.data_ptr(), _stream(stream)),
               "tkv_sparse_select_channels")
        return self.channel_idx

    def prefetch(self, buf: int = 0, stream=None) -> torch.Tensor:
        """Fetch the rows of the current channel list into double-buffer half `buf`."""
        _check(lib().tkv_sparse_prefetch_keys(C.byref(self.layer.desc), C.byref(self.layer.cache), C.byref(self.s1),
                                              self.channel_idx.data_ptr(), self.fetched[buf].data_ptr(),
                                              _stream(stream)), "tkv_sparse_prefetch_keys")
        return self.fetched[buf]

    def estimate_topk(self, q: torch.Tensor, buf: int | None = 0, stream=None):
        """Stage 2 over the fetched buffer `buf`, or (buf=None, resident keys only) in place
        over the channel-major keys."""
        L = self.layer
        d = L.desc
        assert q.dtype == torch.float16 and q.is_cuda and q.is_contiguous()
        if buf is None:
            assert self.resident, "in-place scoring needs device-resident channel-major keys"
            keys, rows = self.keys_cm, d.head_dim
        else:
            keys, rows = self.fetched[buf], d.n_channels
        _check(lib().tkv_sparse_estimate_topk_cm(C.byref(d), C.byref(L.cache), q.data_ptr(),
                                                 self.channel_idx.data_ptr(), keys.data_ptr(), int(rows),
                                                 L.topk_idx.data_ptr(), L.topk_count.data_ptr(),
                                                 L.workspace.data_ptr(), L.workspace_bytes, _stream(stream)),
               "tkv_sparse_estimate_topk_cm")
        return L.topk_idx, L.topk_count


_DTYPES = {torch.float16: 0, torch.bfloat16: 1}


def rope_axes(sections, interleaved: bool = False) -> bytes:
    """The axis of each frequency, for `axis_of`: sections[a] of them belong to axis a, one section after the other, or
    (interleaved) the axes in turn while they have any left."""
    left = [int(n) for n in sections]
    assert all(n >= 0 for n in left)
    if not interleaved:
        return bytes(a for a, n in enumerate(left) for _ in range(n))
    out = []
    while any(left):
        for a, n in enumerate(left):
            if n:
                out.append(a)
                left[a] -= 1
    return bytes(out)


def _rotation(q, k, positions, inv_freq, axis_of, norm, q_weight, k_weight, eps, interleaved, v, out_dtype, n_q_heads=None):
    """What qk_norm_rope and PagedCache.append check and describe alike (q None: its heads count as n_q_heads):
    the descriptor's bytes, its rotary_dim and n_axes."""
    shape_k = k.shape
    t, hkv, ch = shape_k
    dt, at = k.dtype, k.get_device()  # (numbers of devices compare in a third of the time of devices)
    assert k.is_cuda
    sq, sk, sv = (0, 0, 1), k.stride(), (0, 0, 1)
    if q is not None:
        tq, n_q_heads, chq = q.shape
        assert tq == t and chq == ch and q.dtype == dt and q.get_device() == at
        sq = q.stride()
    if v is not None:
        assert v.shape == shape_k and v.dtype == dt and v.get_device() == at
        sv = v.stride()
    assert sq[2] == 1 and sk[2] == 1 and sv[2] == 1
    rot, n_axes = 0, 1
    if inv_freq is not None:
        assert inv_freq.dtype == torch.float32 and inv_freq.dim() == 1 and inv_freq.is_contiguous() and inv_freq.get_device() == at
        assert positions is not None and positions.dtype == torch.int32 and positions.get_device() == at
        assert positions.is_contiguous()
        rot = 2 * inv_freq.shape[0]
        if axis_of is None:
            assert positions.shape == (t,)
        else:
            n_axes, tp = positions.shape
            assert tp == t and 2 * len(axis_of) == rot, "axis_of: an axis for every frequency"
    for w in (q_weight, k_weight):
        assert w is None or (w.shape == (ch,) and w.is_contiguous() and w.dtype == dt and w.get_device() == at)
    # (an axis of one element: torch leaves its stride to chance)
    by_t, by_q, by_k = t > 1, n_q_heads > 1, hkv > 1
    return _ROPE_DESC.pack(_ROPE_DESC.size, n_q_heads, hkv, ch, _DTYPES.get(dt, -1), _DTYPES.get(out_dtype, -1), norm, eps, rot, interleaved,
                           by_t * sq[0], by_q * sq[1], by_t * sk[0], by_k * sk[1], by_t * sv[0], by_k * sv[1]), rot, n_axes


def qk_norm_rope(q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor | None, inv_freq: torch.Tensor | None, *,
                 v: torch.Tensor | None = None, norm: bool = False, q_weight: torch.Tensor | None = None,
                 k_weight: torch.Tensor | None = None, eps: float = 1e-6, interleaved: bool = False, axis_of=None,
                 out_dtype: torch.dtype | None = None, q_out: torch.Tensor | None = None,
                 k_out: torch.Tensor | None = None, v_out: torch.Tensor | None = None, stream=None):
    """tkv_qk_norm_rope: q [T, Hq, 128], k, v [T, Hkv, 128] (fp16 or bf16, views of one fused projection
    allowed), positions int32 [T], inv_freq float32 [R/2] (None: no rotation) -> contiguous (q_out, k_out, v_out or
    None) in out_dtype (default: the inputs').  With axis_of (bytes or small numbers, an axis for every frequency; see rope_axes) positions
    are int32 [axes, T]: tkv_qk_norm_rope_axes."""
    shape_q, at = q.shape, q.get_device()
    handle = _handle(at, stream)
    if axis_of is not None:
        axis_of = bytes(axis_of)
    if out_dtype is None:
        out_dtype = next((x.dtype for x in (q_out, k_out, v_out) if x is not None), q.dtype)
    desc, rot, n_axes = _rotation(q, k, positions, inv_freq, axis_of, norm, q_weight, k_weight, eps, interleaved, v, out_dtype)
    q_out = _given(q_out, q, out_dtype, at, stream)
    k_out = _given(k_out, k, out_dtype, at, stream)
    if v is not None:
        v_out = _given(v_out, v, out_dtype, at, stream)
    else:
        assert v_out is None
    pos, freq = (positions.data_ptr(), inv_freq.data_ptr()) if rot else (0, 0)
    outs = q_out.data_ptr(), k_out.data_ptr(), _ptr(v_out), handle
    if axis_of is None:
        _check(lib().tkv_qk_norm_rope(desc, shape_q[0], q.data_ptr(), k.data_ptr(), _ptr(v), pos, freq, _ptr(q_weight),
                                      _ptr(k_weight), *outs), "tkv_qk_norm_rope")
    else:
        _check(lib().tkv_qk_norm_rope_axes(desc, shape_q[0], q.data_ptr(), k.data_ptr(), _ptr(v), pos, freq, axis_of, n_axes,
                                           _ptr(q_weight), _ptr(k_weight), *outs), "tkv_qk_norm_rope_axes")
    return q_out, k_out, v_out


class PagedCache:
    """A pool of pages that hold keys and values of many sequences, in 16 bits or as microscaled 4-bit floating-point numbers
    (tkv_paged_append, tkv_paged_gather, tkv_paged_attn).  Which pages are whose is the caller's: token t of a sequence whose pages are
    `row` is at slot row[t // page_size] * page_size + t % page_size.  Slots, tables and lengths are device tensors, so a captured decode
    step replays over a cache that grows.  Streams, threads and captured graphs may use one object at the same time (each stream and graph
    has a workspace of its own); calls that write slots and calls that read them are the caller's to order.

    k_pages, v_pages: the pages, where they are the caller's: [n_pages, Hkv, page_size, 128] of dtype (views with any strides whose rows do
    not overlap), or with 4 bits uint8 [n_pages, Hkv, 68 * page_size]; made here (zeros) from n_pages otherwise."""

    def __init__(self, *, n_q_heads=32, n_kv_heads=8, head_dim=128, dtype=torch.float16, bits=16, page_size=64, n_pages=None,
                 k_pages: torch.Tensor | None = None, v_pages: torch.Tensor | None = None, device="cuda:0"):
        assert (k_pages is None) == (v_pages is None)
        if k_pages is None:
            dev = _require_gpu(device)
            row = (page_size, head_dim) if bits == 16 else (68 * page_size,)
            k_pages, v_pages = (torch.zeros(n_pages, n_kv_heads, *row, dtype=dtype if bits == 16 else torch.uint8, device=dev)
                                for _ in range(2))
        assert n_pages is None or n_pages == k_pages.shape[0]
        strides = []
        for x in (k_pages, v_pages):
            assert x.is_cuda and x.get_device() == k_pages.get_device()
            if bits == 16:
                assert x.dtype == dtype and tuple(x.shape) == (k_pages.shape[0], n_kv_heads, page_size, head_dim) and x.stride(3) == 1
                strides.append((C.c_int64 * 3)(*(x.stride(i) if x.shape[i] > 1 else 0 for i in range(3))))
            else:
                assert x.dtype == torch.uint8 and tuple(x.shape) == (k_pages.shape[0], n_kv_heads, 68 * page_size) and x.is_contiguous()
                strides.append((C.c_int64 * 3)())
        self.desc = PagedDesc(C.sizeof(PagedDesc), n_q_heads, n_kv_heads, head_dim, _DTYPES.get(dtype, -1), bits, page_size,
                              k_pages.shape[0], *strides)
        ws = C.c_size_t()
        _check(lib().tkv_paged_attn_sizes(C.byref(self.desc), C.byref(ws)), "tkv_paged_attn_sizes")
        self.workspace_bytes = int(ws.value)
        self.k_pages, self.v_pages, self.dtype = k_pages, v_pages, dtype
        self.device, self._at = k_pages.device, k_pages.get_device()
        self._pages = k_pages.data_ptr(), v_pages.data_ptr()
        self._desc_at = C.addressof(self.desc)
        self._rows = (n_q_heads, head_dim), (n_kv_heads, head_dim)
        self._none = torch.empty(0, dtype=dtype, device=self.device)  # (its new_empty spares half a microsecond of torch.empty's two)
        self._workspaces = _Workspaces(self.workspace_bytes, torch.device("cuda", self._at), at_once=False, zeros=12288)  # (a cache that is only filled needs none)

    def _slots(self, slots, t):
        assert slots.dtype == torch.int32 and slots.shape == (t,) and slots.is_contiguous() and slots.get_device() == self._at

    def append(self, q: torch.Tensor | None, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor,
               positions: torch.Tensor | None = None, inv_freq: torch.Tensor | None = None, *, axis_of=None, norm: bool = False,
               q_weight: torch.Tensor | None = None, k_weight: torch.Tensor | None = None, eps: float = 1e-6, interleaved: bool = False,
               q_out: torch.Tensor | None = None, k_out: torch.Tensor | None = None, stream=None):
        """tkv_paged_append: q [T, Hq, 128], k, v [T, Hkv, 128] and the rotation as for qk_norm_rope; k and v go to slots (int32 [T],
        below 0: nowhere).  Returns q_out [T, Hq, 128] (None without q); k_out [T, Hkv, 128], where given, receives the turned keys
        too."""
        t, at = k.shape[0], self._at
        assert k.get_device() == at and v is not None and k.shape[1:] == self._rows[1] and (q is None or q.shape[1:] == self._rows[0])
        handle = _handle(at, stream)
        self._slots(slots, t)
        if axis_of is not None:
            axis_of = bytes(axis_of)
        dt = self.dtype
        desc, rot, n_axes = _rotation(q, k, positions, inv_freq, axis_of, norm, q_weight, k_weight, eps, interleaved, v, dt,
                                      self._rows[0][0])
        if q is not None:
            q_out = _given(q_out, q, dt, at, stream)
        else:
            assert q_out is None
        if k_out is not None:
            _given(k_out, k, dt, at, stream)
        pos, freq = (positions.data_ptr(), inv_freq.data_ptr()) if rot else (0, 0)
        _check(lib().tkv_paged_append(self._desc_at, desc, t, _ptr(q), k.data_ptr(), v.data_ptr(), pos, freq, axis_of,
                                      n_axes, _ptr(q_weight), _ptr(k_weight), slots.data_ptr(), _ptr(q_out), _ptr(k_out),
                                      *self._pages, handle), "tkv_paged_append")
        return q_out

    def gather(self, slots: torch.Tensor, k_out: torch.Tensor | None = None, v_out: torch.Tensor | None = None, stream=None):
        """tkv_paged_gather: the tokens at slots (int32 [T], below 0: zeros) as contiguous k, v [T, Hkv, 128]."""
        t = slots.shape[0]
        self._slots(slots, t)
        handle = _handle(self._at, stream)
        shape = t, *self._rows[1]
        for o in (k_out, v_out):
            assert o is None or (o.dtype == self.dtype and o.shape == shape and o.is_contiguous() and o.get_device() == self._at)
        if k_out is None:
            k_out = self._none.new_empty(shape) if stream is None else _new(shape, self.dtype, self.device, stream)
        if v_out is None:
            v_out = torch.empty_like(k_out) if stream is None else _new(shape, self.dtype, self.device, stream)
        _check(lib().tkv_paged_gather(self._desc_at, *self._pages, t, slots.data_ptr(), k_out.data_ptr(), v_out.data_ptr(), handle),
               "tkv_paged_gather")
        return k_out, v_out

    def attend(self, q: torch.Tensor, sm_scale: float, page_table: torch.Tensor, k_lens: torch.Tensor, *,
               q_starts: torch.Tensor | None = None, max_q_len: int | None = None, out: torch.Tensor | None = None,
               lse: bool | torch.Tensor = False, stream=None):
        """tkv_paged_attn: q [T, Hq, 128]; page_table int32 [B, pages], k_lens int32 [B]: each sequence's pages and tokens, the queries'
        own among them; q_starts int32 [B + 1]: where each sequence's rows of q begin, max_q_len of them at most (rows beyond that are
        of no sequence; both None: row b is sequence b's only one).  Returns out [T, Hq, 128], or (out, lse [T, Hq]) where lse is True or a
        float32 tensor.  Rows of no sequence are left as they were (new outputs have zeros there, and -inf)."""
        t, at = q.shape[0], self._at
        b, each = page_table.shape
        assert q.dtype == self.dtype and q.shape[1:] == self._rows[0] and q.is_contiguous() and q.get_device() == at
        handle = _handle(at, stream)
        assert page_table.dtype == torch.int32 and page_table.is_contiguous() and page_table.get_device() == at
        assert k_lens.dtype == torch.int32 and k_lens.shape == (b,) and k_lens.is_contiguous() and k_lens.get_device() == at
        if q_starts is None:
            assert t == b and max_q_len in (None, 1)
            max_q_len = 1
        else:
            assert max_q_len is not None, "max_q_len: the most queries of a sequence"
            max_q_len = min(int(max_q_len), max(t, 1))  # (a number beyond 32 bits would be another)
            assert q_starts.dtype == torch.int32 and q_starts.shape == (b + 1,) and q_starts.is_contiguous() and q_starts.get_device() == at
        new_lse = lse is True
        clear = q_starts is not None and out is None and (new_lse or not isinstance(lse, torch.Tensor))  # (by the call itself)
        fill = q_starts is not None and not clear
        if out is None:
            out = _new(q.shape, q.dtype, q.device, stream, 0.0) if fill else _like(q, q.dtype, stream)
        else:
            assert out.dtype == q.dtype and out.shape == q.shape and out.is_contiguous() and out.get_device() == at
        if new_lse:
            if stream is None and not fill:
                lse = q.new_empty((t, self._rows[0][0]), dtype=torch.float32)
            else:
                lse = _new(q.shape[:2], torch.float32, q.device, stream, -float("inf") if fill else None)
        elif lse is False or lse is None:
            lse = None
        else:
            assert lse.dtype == torch.float32 and lse.shape == q.shape[:2] and lse.is_contiguous() and lse.get_device() == at
        with self._workspaces.lock:
            workspace = self._workspaces.of(handle, stream)
            status = lib().tkv_paged_attn(self._desc_at, *self._pages, b, t, max_q_len, q.data_ptr(), out.data_ptr(), _ptr(lse),
                                          page_table.data_ptr(), each, k_lens.data_ptr(), _ptr(q_starts), clear, float(sm_scale),
                                          workspace.data_ptr(), self.workspace_bytes, handle)
        _check(status, "tkv_paged_attn")
        return out if lse is None else (out, lse)


class PromptAttention:
    """Attention over whole prompts, packed sequences and chunks (tkv_prompt_attn): the workspaces and the call.  Streams, threads and
    captured graphs may use one object at the same time (each stream and graph has a workspace of its own, 32.5 MiB)."""

    def __init__(self, *, n_q_heads=32, n_kv_heads=8, head_dim=128, dtype=torch.float16, causal=True, batch=1,
                 device="cuda:0"):
        dev = _require_gpu(device)
        self.desc = PromptDesc(C.sizeof(PromptDesc), n_q_heads, n_kv_heads, head_dim, _DTYPES.get(dtype, -1), int(causal), batch, 0)
        ws = C.c_size_t()
        _check(lib().tkv_prompt_attn_sizes(C.byref(self.desc), C.byref(ws)), "tkv_prompt_attn_sizes")
        self.workspace_bytes = int(ws.value)
        self._at = torch.cuda.current_device() if dev.index is None else dev.index
        self._workspaces = _Workspaces(self.workspace_bytes, torch.device("cuda", self._at))
        self.dtype = dtype
        self.device = dev
        self._q_row, self._k_row = (n_q_heads, head_dim), (n_kv_heads, head_dim)
        self._ints, self._lens_bytes = C.c_int32 * (4 * batch), 4 * batch

    @property
    def workspace(self) -> torch.Tensor:
        """That of the current stream's calls."""
        return self._workspaces.of(_stream(None))

    def attend(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, sm_scale: float, q_lens, k_lens=None, *,
               q_starts=None, k_starts=None, out: torch.Tensor | None = None, lse: bool | torch.Tensor = False, stream=None):
        """q [Tq, Hq, 128], k, v [Tk, Hkv, 128] (views of wider rows allowed); q_lens, k_lens (default: q_lens): tokens of
        every sequence, one after the other unless q_starts / k_starts say where each begins (sequences may share keys, not
        queries).  out: [Tq, Hq, 128], a view too, but not one whose rows overlap.  Returns out
        [Tq, Hq, 128], or (out, lse [Tq, Hq]) where lse is True or a float32 tensor.  Rows of no sequence are left as they
        were (a new out has zeros there)."""
        d, n = self.desc, self.desc.batch
        rows_q, rows_k = q.shape[0], k.shape[0]
        assert q.is_cuda and k.shape == v.shape and q.shape[1:] == self._q_row and k.shape[1:] == self._k_row
        assert q.dtype == k.dtype == v.dtype == self.dtype
        assert q.get_device() == k.get_device() == v.get_device() == self._at
        _on_current(q, stream)

        def ints(x, what):
            x = [*map(int, x)]
            assert len(x) == n and min(x) >= 0, f"{what}: {n} numbers, none below 0"
            return x

        def begin(starts, lens, rows, what):  # (one after the other unless given)
            starts = [0, *itertools.accumulate(lens[:-1])] if starts is None else ints(starts, what)
            assert max(map(operator.add, starts, lens)) <= rows, "a sequence reaches past the tensor's rows"
            return starts

        q_lens = ints(q_lens, "q_lens")
        k_lens = q_lens if k_lens is None else ints(k_lens, "k_lens")
        whole = q_starts is None and sum(q_lens) == rows_q  # every row is some sequence's
        lens = self._ints(*begin(q_starts, q_lens, rows_q, "q_starts"), *q_lens, *begin(k_starts, k_lens, rows_k, "k_starts"), *k_lens)
        by = self._lens_bytes
        if out is None:
            out = _new(q.shape, q.dtype, q.device, stream, None if whole else 0.0)
        else:
            assert out.dtype == q.dtype and out.shape == q.shape and out.device == q.device
        if lse is True:
            lse = _new((rows_q, d.n_q_heads), torch.float32, q.device, stream, None if whole else -float("inf"))
        elif lse is False or lse is None:
            lse = None
        else:
            assert lse.dtype == torch.float32 and lse.shape == q.shape[:2] and lse.is_contiguous() and lse.device == q.device
        (qt, qh, qc), (kt, kh, kc), (vt, vh, vc), (ot, oh, oc) = q.stride(), k.stride(), v.stride(), out.stride()
        assert qc == kc == vc == oc == 1
        # (an axis of one element: torch leaves its stride to chance)
        by_q, by_k, by_qh, by_kh = rows_q > 1, rows_k > 1, d.n_q_heads > 1, d.n_kv_heads > 1
        d = PromptDesc.from_buffer_copy(d)  # (this call's strides: another thread's call may be in the library with its own)
        d.strides[:] = (by_q * qt, by_qh * qh, by_k * kt, by_kh * kh, by_k * vt, by_kh * vh, by_q * ot, by_qh * oh)
        handle = _stream(stream)
        with self._workspaces.lock:
            workspace = self._workspaces.of(handle, stream)
            status = lib().tkv_prompt_attn(C.byref(d), q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), _ptr(lse), lens,
                                           C.byref(lens, by), C.byref(lens, 2 * by), C.byref(lens, 3 * by), float(sm_scale),
                                           workspace.data_ptr(), self.workspace_bytes, handle)
        _check(status, "tkv_prompt_attn")
        return out if lse is None else (out, lse)


class DensePreference:
    """Offline identification of a layer (tkv_dense_preference, tkv_classify_layer)."""

    def __init__(self, *, n_q_heads=32, n_kv_heads=8, head_dim=128, n_q=64, top_k=1024, capacity, batch=1,
                 device="cuda:0"):
        dev = _require_gpu(device)
        self.desc = PrefDesc(C.sizeof(PrefDesc), n_q_heads, n_kv_heads, head_dim, n_q, top_k, capacity, batch)
        ws = C.c_size_t()
        _check(lib().tkv_dense_preference_sizes(C.byref(self.desc), C.byref(ws)), "tkv_dense_preference_sizes")
        self.workspace_bytes = int(ws.value)
        self.workspace = torch.zeros(self.workspace_bytes, dtype=torch.uint8, device=dev)
        self.device = dev

    def score(self, q_last: torch.Tensor, k: torch.Tensor, sm_scale: float, stream=None) -> torch.Tensor:
        """q_last fp16 [B, n_q, Hq, D], k fp16 [B, n, Hkv, D] -> float32 [B, Hq] (Eq. 8 per head)."""
        d = self.desc
        for t in (q_last, k):
            assert t.dtype == torch.float16 and t.is_cuda and t.is_contiguous()
        assert tuple(q_last.shape) == (d.batch, d.n_q, d.n_q_heads, d.head_dim)
        assert k.shape[0] == d.batch and tuple(k.shape[2:]) == (d.n_kv_heads, d.head_dim)
        out = torch.empty(d.batch, d.n_q_heads, dtype=torch.float32, device=self.device)
        _check(lib().tkv_dense_preference(C.byref(d), q_last.data_ptr(), k.data_ptr(), int(k.shape[1]),
                                          float(sm_scale), out.data_ptr(), self.workspace.data_ptr(),
                                          self.workspace_bytes, _stream(stream)), "tkv_dense_preference")
        return out

    def classify(self, p_heads: torch.Tensor, tau: float = 0.2):
        """Eq. 9 for one sequence: (True if quantization-friendly, layer score)."""
        p = np.ascontiguousarray(p_heads.detach().float().cpu().numpy().reshape(-1), dtype=np.float32)
        score = C.c_float()
        r = lib().tkv_classify_layer(p.ctypes.data_as(C.POINTER(C.c_float)), int(p.size), int(self.desc.n_q),
                                     float(tau), C.byref(score))
        if r < 0:
            raise TkvError(r, "tkv_classify_layer")
        return bool(r), float(score.value)
