"""ctypes binding of include/ebag_a2a.h and include/gemv_ar.h (same names,
argument marshalling only).

Device buffers may be passed as torch tensors (their ``data_ptr()`` is used)
or as integer device addresses.  The stream defaults to torch's current
stream on the current device.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libebag_a2a.so")

EBAG_F32, EBAG_F16, EBAG_BF16 = 0, 1, 2
EBAG_OK, EBAG_EINVAL, EBAG_EUNSUPPORTED, EBAG_EHIP, EBAG_ETIMEOUT, EBAG_ENOMEM, EBAG_EBUSY = 0, -1, -2, -3, -4, -5, -6


class Opts(ctypes.Structure):
    _fields_ = [
        ("waves_per_wg", ctypes.c_int32),
        ("bags_per_run", ctypes.c_int32),
        ("rows_in_flight", ctypes.c_int32),
        ("persistent_wgs_per_cu", ctypes.c_int32),
        ("release_mode", ctypes.c_int32),
        ("chunk_order", ctypes.c_int32),
        ("self_rank", ctypes.c_int32),
        ("trace", ctypes.c_int32),
        ("check_indices", ctypes.c_int32),
        ("debug_suppress_flag", ctypes.c_int32),
        ("consumer_wgs", ctypes.c_int32),
        ("stream_rows", ctypes.c_int32),
        ("consume_timeout_us", ctypes.c_int64),
        ("pooling_mode", ctypes.c_int32),
        ("slice_granule", ctypes.c_int32),
        ("backward_bags_per_run", ctypes.c_int32),
        ("backward_waves_per_wg", ctypes.c_int32),
        ("table_major", ctypes.c_int32),
        ("consume_nontemporal", ctypes.c_int32),
        ("deliver_wgs", ctypes.c_int32),
        ("deliver_waves_per_wg", ctypes.c_int32),
    ]


class GemvOpts(ctypes.Structure):
    _fields_ = [
        ("tile_rows", ctypes.c_int32),
        ("wgs_per_rank", ctypes.c_int32),
        ("waves_per_wg", ctypes.c_int32),
        ("comm_aware", ctypes.c_int32),
        ("debug_suppress_flag", ctypes.c_int32),
        ("reduce_mode", ctypes.c_int32),
        ("timeout_us", ctypes.c_int64),
    ]


class EbagError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"ebag_a2a error {code}: {msg}")
        self.code = code


_lib = None

_P = ctypes.c_void_p
_SIGS = {
    "ebag_a2a_default_opts": ([_P], ctypes.c_int),
    "ebag_a2a_create": ([_P, ctypes.c_int32, _P, _P, ctypes.c_int32, ctypes.c_int32, ctypes.c_int64, ctypes.c_int32, _P],
                        ctypes.c_int),
    "ebag_a2a_forward": ([_P, _P, _P, _P, _P, ctypes.c_int64, ctypes.c_int32, _P, _P, _P], ctypes.c_int),
    "ebag_a2a_unfused_forward": ([_P, _P, _P, _P, _P, ctypes.c_int64, ctypes.c_int32, _P, _P, _P], ctypes.c_int),
    "ebag_a2a_forward_noalloc": ([ctypes.c_int32, _P, _P, ctypes.c_int32, ctypes.c_int32, _P, _P, _P, _P, _P,
                                  ctypes.c_int64, ctypes.c_int32, _P, _P, _P], ctypes.c_int),
    "ebag_a2a_consume": ([_P, _P, _P, _P, ctypes.c_int64, ctypes.c_int32, ctypes.c_uint32, _P], ctypes.c_int),
    "ebag_a2a_backward": ([_P, _P, _P, ctypes.c_uint32, _P, _P, ctypes.c_int64, ctypes.c_int32, _P, _P], ctypes.c_int),
    "ebag_a2a_deliver": ([_P, _P, _P, _P, ctypes.c_int64, ctypes.c_int32, _P], ctypes.c_int),
    "ebag_a2a_status": ([_P, _P, _P], ctypes.c_int),
    "ebag_a2a_status_ex": ([_P, _P], ctypes.c_int),
    "ebag_a2a_reset": ([_P], ctypes.c_int),
    "ebag_a2a_trace": ([_P, _P, _P, ctypes.c_int64, _P], ctypes.c_int),
    "ebag_a2a_occupancy": ([_P, ctypes.c_int32, _P], ctypes.c_int),
    "ebag_a2a_queue_stream_create": ([_P], ctypes.c_int),
    "ebag_a2a_queue_stream_destroy": ([_P], ctypes.c_int),
    "ebag_a2a_destroy": ([_P], None),
    "ebag_a2a_last_error": ([], ctypes.c_char_p),
    "ebag_a2a_moe_create": ([_P, ctypes.c_int64, ctypes.c_int32, ctypes.c_int32], ctypes.c_int),
    "ebag_a2a_moe_sort": ([_P, _P, ctypes.c_int64, _P, _P, _P, _P], ctypes.c_int),
    "ebag_a2a_moe_dispatch": ([_P, _P, ctypes.c_int64, ctypes.c_int64, ctypes.c_int32, ctypes.c_int64, _P, _P, _P,
                               ctypes.c_int64, _P], ctypes.c_int),
    "ebag_a2a_moe_dispatch_backward": ([_P, _P, ctypes.c_int64, ctypes.c_int64, ctypes.c_int32, ctypes.c_int64, _P, _P,
                                        _P, ctypes.c_int64, _P], ctypes.c_int),
    "ebag_a2a_moe_combine": ([_P, _P, ctypes.c_int64, ctypes.c_int64, ctypes.c_int32, ctypes.c_int64, _P, _P, _P, _P,
                              ctypes.c_int64, _P], ctypes.c_int),
    "ebag_a2a_moe_combine_backward": ([_P, _P, ctypes.c_int64, _P, ctypes.c_int64, ctypes.c_int64, ctypes.c_int32,
                                       ctypes.c_int64, _P, _P, _P, _P, ctypes.c_int64, _P, _P], ctypes.c_int),
    "ebag_a2a_moe_choose_work": ([_P], ctypes.c_int64),
    "ebag_a2a_moe_choose": ([_P, _P, ctypes.c_int64, ctypes.c_int32, ctypes.c_int64, _P, _P, ctypes.c_int32, _P, _P, _P, _P,
                             _P, _P, _P], ctypes.c_int),
    "ebag_a2a_moe_choose_backward": ([_P, _P, ctypes.c_int64, ctypes.c_int32, ctypes.c_int64, _P, ctypes.c_int32, _P, _P, _P,
                                      _P, _P, ctypes.c_int64, _P], ctypes.c_int),
    "ebag_a2a_moe_destroy": ([_P], None),
    "gemv_ar_default_opts": ([_P], ctypes.c_int),
    "gemv_ar_create": ([_P, ctypes.c_int32, ctypes.c_int64, _P, ctypes.c_int32, _P], ctypes.c_int),
    "gemv_ar_forward": ([_P, _P, _P, _P, _P, _P], ctypes.c_int),
    "gemv_ar_unfused_forward": ([_P, _P, _P, _P, _P, _P], ctypes.c_int),
    "gemv_ar_status": ([_P, _P], ctypes.c_int),
    "gemv_ar_reset": ([_P], ctypes.c_int),
    "gemv_ar_launch_info": ([_P, _P], ctypes.c_int),
    "gemv_ar_destroy": ([_P], None),
    "gemv_ar_q4_create": ([_P, ctypes.c_int64, ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                           ctypes.c_int32], ctypes.c_int),
    "gemv_ar_q4_quantize": ([_P, _P, _P, _P, _P, _P], ctypes.c_int),
    "gemv_ar_q4_forward": ([_P, _P, _P, _P, _P, ctypes.c_int64, ctypes.c_int64, _P, ctypes.c_int64, ctypes.c_int32, _P],
                           ctypes.c_int),
    "gemv_ar_q4_experts": ([_P, _P, _P, _P, _P, ctypes.c_int64, ctypes.c_int64, _P, _P, ctypes.c_int32, ctypes.c_int64,
                            _P, ctypes.c_int64, ctypes.c_int32, _P], ctypes.c_int),
    "gemv_ar_q4_destroy": ([_P], None),
    "gemv_ar_q8_create": ([_P, ctypes.c_int64, ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32], ctypes.c_int),
    "gemv_ar_q8_pitch": ([_P], ctypes.c_int64),
    "gemv_ar_q8_quantize": ([_P, _P, _P, _P, _P], ctypes.c_int),
    "gemv_ar_q8_round": ([_P, _P, ctypes.c_int64, ctypes.c_int64, _P, _P, _P], ctypes.c_int),
    "gemv_ar_q8_forward": ([_P, _P, _P, _P, ctypes.c_int64, ctypes.c_int64, _P, _P, _P, ctypes.c_int64, ctypes.c_int32, _P],
                           ctypes.c_int),
    "gemv_ar_q8_experts": ([_P, _P, _P, _P, ctypes.c_int64, ctypes.c_int64, _P, _P, _P, _P, ctypes.c_int32, ctypes.c_int64,
                            _P, ctypes.c_int64, ctypes.c_int32, _P], ctypes.c_int),
    "gemv_ar_q8_destroy": ([_P], None),
}


def symbols():
    """Names of the C ABI entry points this binding expects."""
    return list(_SIGS)


def load(path: str = LIB_PATH):
    """Load the HIP library (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"HIP library {path} not found: build it with `python __graft_entry__.py` "
                           "(there is no CPU fallback)")
    lib = ctypes.CDLL(path)
    for name, (args, res) in _SIGS.items():
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = res
    _lib = lib
    return lib


def last_error() -> str:
    return load().ebag_a2a_last_error().decode()


def _check(rc: int):
    if rc != EBAG_OK:
        raise EbagError(rc, last_error())


def _addr(x) -> Optional[int]:
    if x is None or isinstance(x, int):
        return x
    return x.data_ptr()


_current_stream = None  # the current device's current stream, as an address


def _find_current_stream():
    """torch.cuda.current_stream() builds a stream object, 2.9 us of a call
    that takes 6 in all; torch also has the stream's address alone."""
    import torch
    raw, device = (getattr(torch._C, n, None) for n in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))
    if raw is None or device is None:
        return lambda: torch.cuda.current_stream().cuda_stream
    return lambda: raw(device())


def _stream(stream) -> Optional[int]:
    global _current_stream
    if stream is None:
        if _current_stream is None:
            import torch
            if not torch.cuda.is_initialized():
                return torch.cuda.current_stream().cuda_stream
            _current_stream = _find_current_stream()
        return _current_stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _need(buf, nbytes: int, what: str, i: int = 0):
    """A torch tensor passed as a buffer must hold at least nbytes (raw
    integer addresses are the caller's responsibility).  what: its name, with a
    {} for its position i among several."""
    if buf is None or isinstance(buf, int) or not hasattr(buf, "numel"):
        return
    if buf.numel() * buf.element_size() < nbytes:
        raise ValueError(f"{what.format(i)} holds {buf.numel() * buf.element_size()} bytes, needs {nbytes}")


F32 = ("float32",)
I32 = ("int32",)
I64 = ("int64",)
FLAG_TYPES = ("int32", "uint32")
_DTYPES = {}  # dtype -> its name


def _dtype_name(dt) -> str:
    name = _DTYPES.get(dt)
    if name is None:
        name = _DTYPES[dt] = str(dt).replace("torch.", "")
    return name


def _validate(*specs):
    """Every torch tensor handed to a kernel must be contiguous, of the
    element type the C ABI reads and on the GPU.  specs: (tensors, name,
    allowed dtype names or None, element bytes or None), the name with a {} for
    a tensor's position among several; None and raw integer addresses are
    skipped (those are the caller's responsibility).  Layout and type are
    checked for every tensor before the device of any.  The checks run on every
    call, a few hundred tensors of them for a large plan: names are put together
    only for an error."""
    off_gpu = None
    for xs, what, kinds, elt in specs:
        for i, x in enumerate(xs):
            if x is None or isinstance(x, int):
                continue
            try:
                contiguous = x.is_contiguous()
            except AttributeError:
                continue
            if not contiguous:
                raise ValueError(f"{what.format(i)} must be contiguous")
            if kinds is not None and _dtype_name(x.dtype) not in kinds:
                raise ValueError(f"{what.format(i)} must be {' or '.join(kinds)}, not {_dtype_name(x.dtype)}")
            if elt is not None and x.element_size() != elt:
                raise ValueError(f"{what.format(i)} must have {elt}-byte elements, not {x.element_size()}-byte "
                                 f"{_dtype_name(x.dtype)}")
            if off_gpu is None and not x.is_cuda:
                off_gpu = what.format(i), x.device
    if off_gpu is not None:
        raise ValueError(f"{off_gpu[0]} must be a GPU tensor, not one on {off_gpu[1]}")


def _elt(dtype) -> int:
    return 4 if int(dtype) == EBAG_F32 else 2


def queue_stream():
    """A torch stream on a hardware queue of its own (ebag_a2a_queue_stream_create)."""
    import torch
    s = ctypes.c_void_p()
    _check(load().ebag_a2a_queue_stream_create(ctypes.byref(s)))
    return torch.cuda.ExternalStream(s.value)


def queue_stream_destroy(stream):
    """Drain and destroy a stream from queue_stream() (ebag_a2a_queue_stream_destroy)."""
    _check(load().ebag_a2a_queue_stream_destroy(_stream(stream)))


def default_opts() -> Opts:
    o = Opts()
    _check(load().ebag_a2a_default_opts(ctypes.byref(o)))
    return o


NOALLOC_MAX_TABLES, NOALLOC_MAX_FLAGS = 1024, 65536


def forward_noalloc(rows, dims, dtype, chunk_samples, tables, indices, offsets, weights, B, R, send, flags,
                    stream=None, **opts):
    """Plan-free fused forward (``ebag_a2a_forward_noalloc``): the same result
    as ``Plan(rows, dims, dtype, chunk_samples, ..., **opts).forward(...)``,
    with the plan's device memory in the library's static per-GPU array."""
    lib = load()
    o = default_opts()
    for k, v in opts.items():
        if not hasattr(o, k):
            raise TypeError(f"unknown option {k}")
        setattr(o, k, int(v))
    T = len(rows)
    if len(dims) != T or len(tables) != T:
        raise ValueError("rows, dims and tables must have one entry per table")
    n_flags = (int(B) // int(chunk_samples)) * (T if o.slice_granule == 1 else 1)
    _need(send, 4 * int(B) * sum(int(d) for d in dims), "send buffer")
    _need(flags, 4 * n_flags, "flags")
    _need(offsets, 8 * (T * int(B) + 1), "offsets")
    _validate((tables, "table {}", None, _elt(dtype)), ((indices,), "indices", I32, None),
              ((offsets,), "offsets", I64, None), ((weights,), "weights", F32, None),
              ((send,), "send buffer", F32, None), ((flags,), "flags", FLAG_TYPES, None))
    if hasattr(indices, "numel") and indices.numel() == 0:
        raise ValueError("indices must have a device address: pass a one-element buffer when every bag is empty")
    rows_a = (ctypes.c_int64 * T)(*[int(r) for r in rows])
    dims_a = (ctypes.c_int32 * T)(*[int(d) for d in dims])
    tabs = (ctypes.c_void_p * T)(*[_addr(t) for t in tables])
    _check(lib.ebag_a2a_forward_noalloc(T, rows_a, dims_a, int(dtype), int(chunk_samples), ctypes.byref(o), tabs,
                                        _addr(indices), _addr(offsets), _addr(weights), int(B), int(R), _addr(send),
                                        _addr(flags), _stream(stream)))


class Plan:
    """A plan for T tables (``ebag_a2a_create``); methods mirror the C ABI."""

    def __init__(self, rows: Sequence[int], dims: Sequence[int], dtype: int, chunk_samples: int, max_batch: int,
                 max_ranks: int, **opts):
        lib = load()
        o = default_opts()
        for k, v in opts.items():
            if not hasattr(o, k):
                raise TypeError(f"unknown option {k}")
            setattr(o, k, int(v))
        self.T = len(rows)
        self.dims = [int(d) for d in dims]
        self.C = int(chunk_samples)
        self.elt = _elt(dtype)
        self.opts = o
        rows_a = (ctypes.c_int64 * self.T)(*[int(r) for r in rows])
        dims_a = (ctypes.c_int32 * self.T)(*self.dims)
        h = ctypes.c_void_p()
        _check(lib.ebag_a2a_create(ctypes.byref(h), self.T, rows_a, dims_a, int(dtype), self.C, int(max_batch),
                                   int(max_ranks), ctypes.byref(o)))
        self._h = h
        self._lib = lib
        self._tab_cache = None
        self._empty_idx = None

    def _indices(self, indices):
        """An empty index tensor (every bag empty) has no device address; the
        C ABI takes a valid pointer that is never read, so pass a one-element
        device buffer instead."""
        if hasattr(indices, "numel") and indices.numel() == 0:
            if self._empty_idx is None or self._empty_idx.device != indices.device:
                import torch
                self._empty_idx = torch.zeros(1, dtype=torch.int32, device=indices.device)
            return self._empty_idx.data_ptr()
        return _addr(indices)

    def _tables(self, tables):
        ptrs = [_addr(t) for t in tables]
        if len(ptrs) != self.T:
            raise ValueError(f"expected {self.T} tables, got {len(ptrs)}")
        if self._tab_cache is None or self._tab_cache[0] != ptrs:
            self._tab_cache = (ptrs, (ctypes.c_void_p * self.T)(*ptrs))
        return self._tab_cache[1]

    def _fwd_sizes(self, B, send, flags):
        _need(send, 4 * int(B) * sum(self.dims), "send buffer")
        _need(flags, 4 * self.n_flags(int(B)), "flags")

    def _fwd_types(self, tables, indices, offsets, weights, send, flags):
        _validate((tables, "table {}", None, self.elt), ((indices,), "indices", I32, None),
                  ((offsets,), "offsets", I64, None), ((weights,), "weights", F32, None),
                  ((send,), "send buffer", F32, None), ((flags,), "flags", FLAG_TYPES, None))

    def forward(self, tables, indices, offsets, weights, B, R, send, flags, stream=None):
        self._fwd_sizes(B, send, flags)
        _need(offsets, 8 * (self.T * int(B) + 1), "offsets")
        self._fwd_types(tables, indices, offsets, weights, send, flags)
        _check(self._lib.ebag_a2a_forward(self._h, self._tables(tables), self._indices(indices),
                                          _addr(offsets), _addr(weights), int(B), int(R), _addr(send),
                                          _addr(flags), _stream(stream)))

    def unfused_forward(self, tables, indices, offsets, weights, B, R, send, flags, stream=None):
        self._fwd_sizes(B, send, flags)
        _need(offsets, 8 * (self.T * int(B) + 1), "offsets")
        self._fwd_types(tables, indices, offsets, weights, send, flags)
        _check(self._lib.ebag_a2a_unfused_forward(self._h, self._tables(tables), self._indices(indices),
                                                  _addr(offsets), _addr(weights), int(B), int(R),
                                                  _addr(send), _addr(flags), _stream(stream)))

    def consume(self, send, flags, recv, B, R, expected_epoch, stream=None):
        self._fwd_sizes(B, send, flags)
        _need(recv, 4 * int(B) * sum(self.dims), "recv buffer")
        _validate(((send,), "send buffer", F32, None), ((flags,), "flags", FLAG_TYPES, None),
                  ((recv,), "recv buffer", F32, None))
        _check(self._lib.ebag_a2a_consume(self._h, _addr(send), _addr(flags), _addr(recv), int(B), int(R),
                                          int(expected_epoch) & 0xFFFFFFFF, _stream(stream)))

    def backward(self, grad, offsets, weights, B, R, values, grad_flags=None, expected_epoch=0, stream=None):
        self._fwd_sizes(B, grad, grad_flags)
        _need(offsets, 8 * (self.T * int(B) + 1), "offsets")
        _validate(((grad,), "gradient", F32, None), ((grad_flags,), "gradient flags", FLAG_TYPES, None),
                  ((offsets,), "offsets", I64, None), ((weights,), "weights", F32, None),
                  ((values,), "values", F32, None))
        _check(self._lib.ebag_a2a_backward(self._h, _addr(grad), _addr(grad_flags), int(expected_epoch) & 0xFFFFFFFF,
                                           _addr(offsets), _addr(weights), int(B), int(R), _addr(values),
                                           _stream(stream)))

    def deliver(self, src, dst, flags, B, R, stream=None):
        self._fwd_sizes(B, src, flags)
        _need(dst, 4 * int(B) * sum(self.dims), "destination buffer")
        _validate(((src,), "source buffer", F32, None), ((dst,), "destination buffer", F32, None),
                  ((flags,), "flags", FLAG_TYPES, None))
        _check(self._lib.ebag_a2a_deliver(self._h, _addr(src), _addr(dst), _addr(flags), int(B), int(R),
                                          _stream(stream)))

    def status(self):
        """(timed_out, first_missing_flag); synchronises the device."""
        s = (ctypes.c_int32 * 4)()
        _check(self._lib.ebag_a2a_status_ex(self._h, s))
        return s[0], s[1]

    def status_ex(self):
        s = (ctypes.c_int32 * 4)()
        _check(self._lib.ebag_a2a_status_ex(self._h, s))
        return tuple(s)

    def reset(self):
        _check(self._lib.ebag_a2a_reset(self._h))

    def n_flags(self, B):
        """Flag count of a forward over B samples (B / C, times T per-table)."""
        return (B // self.C) * (self.T if self.opts.slice_granule == 1 else 1)

    def trace(self, n):
        import numpy as np
        rel = np.zeros(n, dtype=np.uint64)
        drn = np.zeros(n, dtype=np.uint64)
        tpu = ctypes.c_double()
        _check(self._lib.ebag_a2a_trace(self._h, rel.ctypes.data, drn.ctypes.data, n, ctypes.byref(tpu)))
        return rel, drn, tpu.value

    def occupancy(self, weighted=False):
        """(max resident WGs per CU, CUs, threads per WG, bags per run) of the fused kernel."""
        s = (ctypes.c_int32 * 4)()
        _check(self._lib.ebag_a2a_occupancy(self._h, int(bool(weighted)), s))
        return tuple(s)

    def close(self):
        if getattr(self, "_h", None):
            self._lib.ebag_a2a_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


ROW_TYPES = {"float32": EBAG_F32, "float16": EBAG_F16, "bfloat16": EBAG_BF16}


def _refuse(*specs):
    """Says what is wrong with tensors that _fit() turned down.  specs: (tensor,
    name, allowed dtype names, bytes needed)."""
    _validate(*(((x,), what, kinds, None) for x, what, kinds, _ in specs))
    for x, what, _, nbytes in specs:
        _need(x, nbytes, what)
    raise ValueError(f"unusable tensors among {', '.join(what for _, what, _, _ in specs)}")


def _fit(x, dtype, count: int) -> bool:
    """Whether a tensor is one of at least `count` elements that a kernel can
    take: _validate() and _need() in one go, for calls of a few microseconds."""
    return x.dtype is dtype and x.is_cuda and x.is_contiguous() and x.numel() >= count


def _matrix(x, rows: int, cols: int, kind: Optional[str], what: str):
    """(address, row step in elements, type name) of a matrix on the GPU: a
    tensor [rows or more, cols] whose rows are contiguous, one step apart."""
    name = _DTYPES.get(x.dtype) or _dtype_name(x.dtype)
    if name not in ROW_TYPES or (kind is not None and name != kind):
        raise ValueError(f"{what} must be {kind or ' or '.join(ROW_TYPES)}, not {name}")
    shape = x.shape
    if len(shape) != 2 or shape[0] < rows or shape[1] != cols:
        raise ValueError(f"{what} must be [{rows}, {cols}], not {list(shape)}")
    step, inner = x.stride()
    if shape[0] <= 1:
        step = cols
    if (inner != 1 and cols > 1) or step < cols:
        raise ValueError(f"{what} must have contiguous rows that do not overlap")
    if not x.is_cuda:
        raise ValueError(f"{what} must be a GPU tensor, not one on {x.device}")
    return x.data_ptr(), step, name


class MoePerm:
    """A plan for sorting tokens by expert (``ebag_a2a_moe_create``): up to
    max_tokens tokens of `choices` choices each, `experts` experts.  Methods
    mirror the C ABI and take torch tensors: choices and places int32
    [tokens, choices], offsets int32 [experts + 1], src int32 [tokens *
    choices], weights float32 [tokens, choices], rows float32, float16 or
    bfloat16 with any step between them."""

    def __init__(self, max_tokens: int, choices: int, experts: int):
        lib = load()
        h = ctypes.c_void_p()
        _check(lib.ebag_a2a_moe_create(ctypes.byref(h), int(max_tokens), int(choices), int(experts)))
        self._h = h
        self._lib = lib
        self._shape(choices, experts)

    def _shape(self, choices, experts):
        import torch
        self.choices, self.experts = int(choices), int(experts)
        self._i32, self._f32 = torch.int32, torch.float32
        self._flags = (torch.bool, torch.uint8)
        self.choose_work = 32 + 512 * (self.experts + 1)  # ebag_a2a_moe_choose_work

    def _places(self, offsets, pos, *weights) -> int:
        """Checks what every call over rows shares; the number of tokens.
        weights: the call's float32 [tokens, choices] tensors."""
        n = pos.numel()
        tokens = n // self.choices
        if n != tokens * self.choices:
            raise ValueError(f"pos must be [tokens, {self.choices}], not {list(pos.shape)}")
        ok = _fit(offsets, self._i32, self.experts + 1) and _fit(pos, self._i32, 0)
        for w in weights:
            ok = ok and _fit(w, self._f32, n)
        if not ok:
            _refuse((offsets, "offsets", I32, 4 * (self.experts + 1)), (pos, "pos", I32, 0),
                    *((w, what, F32, 4 * n) for w, what in zip(weights, ("weights", "dweights"))))
        return tokens

    def _live(self, live, n):
        """live: None, or one truth value of a byte for each of n tokens."""
        if live is not None and not (live.dtype in self._flags and live.is_cuda and live.is_contiguous() and live.numel() >= n):
            _refuse((live, "live", ("bool", "uint8"), n))
        return _addr(live)

    def choose(self, logits, ids, weights, counts=None, sums=None, losses=None, work=None, bias=None, live=None,
               normalise=True, stream=None):
        """ebag_a2a_moe_choose.  counts, sums, losses and work (float32
        [choose_work]) go together; live: bool or uint8 [tokens]."""
        n, k, E = logits.shape[0], self.choices, self.experts
        pl, ldl, kind = _matrix(logits, n, E, None, "logits")
        ok = _fit(ids, self._i32, n * k) and _fit(weights, self._f32, n * k) and (bias is None or _fit(bias, self._f32, E))
        totals = counts is not None or sums is not None or losses is not None or work is not None
        if totals:
            if counts is None or sums is None or losses is None or work is None:
                raise ValueError("counts, sums, losses and work go together: all of them or none")
            ok = (ok and _fit(counts, self._i32, E + 1) and _fit(sums, self._f32, E + 1) and _fit(losses, self._f32, 2) and
                  _fit(work, self._f32, self.choose_work))
        if not ok:
            _refuse((ids, "ids", I32, 4 * n * k), (weights, "weights", F32, 4 * n * k), (bias, "bias", F32, 4 * E),
                    (counts, "counts", I32, 4 * (E + 1)), (sums, "sums", F32, 4 * (E + 1)), (losses, "losses", F32, 8),
                    (work, "work", F32, 4 * self.choose_work))
        _check(self._lib.ebag_a2a_moe_choose(self._h, pl, ldl, ROW_TYPES[kind], n, _addr(bias), self._live(live, n),
                                             int(bool(normalise)), ids.data_ptr(), weights.data_ptr(), _addr(counts),
                                             _addr(sums), _addr(losses), _addr(work), _stream(stream)))

    def choose_backward(self, logits, ids, dweights, dlogits, counts=None, dlosses=None, live=None, normalise=True,
                        stream=None):
        """ebag_a2a_moe_choose_backward.  dweights may be None, and dlosses (then
        counts, too)."""
        n, k, E = logits.shape[0], self.choices, self.experts
        pl, ldl, kind = _matrix(logits, n, E, None, "logits")
        pd, ldd, _ = _matrix(dlogits, n, E, kind, "dlogits")
        ok = dweights is None or (ids is not None and _fit(ids, self._i32, n * k) and _fit(dweights, self._f32, n * k))
        if dlosses is not None:
            ok = ok and _fit(dlosses, self._f32, 2) and counts is not None and _fit(counts, self._i32, E + 1)
        if not ok:
            if dweights is not None and ids is None or dlosses is not None and counts is None:
                raise ValueError("dweights need ids, dlosses need counts")
            _refuse((ids, "ids", I32, 4 * n * k), (dweights, "dweights", F32, 4 * n * k), (dlosses, "dlosses", F32, 8),
                    (counts, "counts", I32, 4 * (E + 1)))
        _check(self._lib.ebag_a2a_moe_choose_backward(self._h, pl, ldl, ROW_TYPES[kind], n, self._live(live, n),
                                                      int(bool(normalise)), _addr(ids), _addr(dweights), _addr(counts),
                                                      _addr(dlosses), pd, ldd, _stream(stream)))

    def sort(self, experts_of, offsets, pos, src, stream=None):
        n, i32 = experts_of.numel(), self._i32
        if n % self.choices:
            raise ValueError(f"experts_of must be [tokens, {self.choices}], not {list(experts_of.shape)}")
        if not (_fit(experts_of, i32, 0) and _fit(offsets, i32, self.experts + 1) and _fit(pos, i32, n) and _fit(src, i32, n)):
            _refuse((experts_of, "experts_of", I32, 0), (offsets, "offsets", I32, 4 * (self.experts + 1)),
                    (pos, "pos", I32, 4 * n), (src, "src", I32, 4 * n))
        _check(self._lib.ebag_a2a_moe_sort(self._h, experts_of.data_ptr(), n // self.choices, offsets.data_ptr(),
                                           pos.data_ptr(), src.data_ptr(), _stream(stream)))

    def dispatch(self, x, offsets, pos, xs, stream=None):
        n = self._places(offsets, pos)
        dim = x.shape[-1]
        px, ldx, kind = _matrix(x, n, dim, None, "x")
        pxs, ldxs, _ = _matrix(xs, n * self.choices, dim, kind, "xs")
        _check(self._lib.ebag_a2a_moe_dispatch(self._h, px, ldx, dim, ROW_TYPES[kind], n, offsets.data_ptr(),
                                               pos.data_ptr(), pxs, ldxs, _stream(stream)))

    def dispatch_backward(self, dxs, offsets, pos, dx, stream=None):
        n = self._places(offsets, pos)
        dim = dxs.shape[-1]
        ps, lds, kind = _matrix(dxs, n * self.choices, dim, None, "dxs")
        pd, ldd, _ = _matrix(dx, n, dim, kind, "dx")
        _check(self._lib.ebag_a2a_moe_dispatch_backward(self._h, ps, lds, dim, ROW_TYPES[kind], n, offsets.data_ptr(),
                                                        pos.data_ptr(), pd, ldd, _stream(stream)))

    def combine(self, ys, offsets, pos, weights, out, stream=None):
        n = self._places(offsets, pos, weights)
        dim = ys.shape[-1]
        py, ldy, kind = _matrix(ys, n * self.choices, dim, None, "ys")
        po, ldo, _ = _matrix(out, n, dim, kind, "out")
        _check(self._lib.ebag_a2a_moe_combine(self._h, py, ldy, dim, ROW_TYPES[kind], n, offsets.data_ptr(),
                                              pos.data_ptr(), weights.data_ptr(), po, ldo, _stream(stream)))

    def combine_backward(self, dout, ys, offsets, pos, weights, dys, dweights, stream=None):
        n = self._places(offsets, pos, weights, dweights)
        dim = ys.shape[-1]
        pd, ldd, kind = _matrix(dout, n, dim, None, "dout")
        py, ldy, _ = _matrix(ys, n * self.choices, dim, kind, "ys")
        ps, lds, _ = _matrix(dys, n * self.choices, dim, kind, "dys")
        _check(self._lib.ebag_a2a_moe_combine_backward(self._h, pd, ldd, py, ldy, dim, ROW_TYPES[kind], n,
                                                       offsets.data_ptr(), pos.data_ptr(), weights.data_ptr(), ps, lds,
                                                       dweights.data_ptr(), _stream(stream)))

    def close(self):
        if getattr(self, "_h", None):
            self._lib.ebag_a2a_moe_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def gemv_default_opts() -> GemvOpts:
    o = GemvOpts()
    _check(load().gemv_ar_default_opts(ctypes.byref(o)))
    return o


class GemvAR:
    """A fused GEMV + AllReduce plan (``gemv_ar_create``) for R ranks; methods
    mirror the C ABI.  A, x, y are sequences of R device buffers."""

    def __init__(self, R: int, M: int, K: Sequence[int], dtype: int, **opts):
        lib = load()
        o = gemv_default_opts()
        for k, v in opts.items():
            if not hasattr(o, k):
                raise TypeError(f"unknown option {k}")
            setattr(o, k, int(v))
        self.R, self.M, self.K = int(R), int(M), [int(k) for k in K]
        self.elt = _elt(dtype)
        self.opts = o
        ks = (ctypes.c_int64 * len(self.K))(*self.K)
        h = ctypes.c_void_p()
        _check(lib.gemv_ar_create(ctypes.byref(h), self.R, self.M, ks, int(dtype), ctypes.byref(o)))
        self._h = h
        self._lib = lib
        self._P = self.launch_info()[0]
        self._ptrs = ctypes.c_void_p * self.R

    def _arrays(self, A, x, y):
        if not (len(A) == len(x) == len(y) == self.R):
            raise ValueError(f"expected {self.R} buffers each for A, x and y")
        for r in range(self.R):
            _need(A[r], self.M * self.K[r] * self.elt, "A[{}]", r)
            _need(x[r], self.K[r] * self.elt, "x[{}]", r)
        _validate((A, "A[{}]", None, self.elt), (x, "x[{}]", None, self.elt), (y, "y[{}]", F32, None))
        arr = self._ptrs
        return arr(*[_addr(a) for a in A]), arr(*[_addr(v) for v in x]), arr(*[_addr(v) for v in y])

    def _out_sizes(self, y, out_flags):
        for v in y:
            _need(v, 4 * self.M, "output vector")
        _need(out_flags, 4 * self.R * self._P, "out_flags")
        _validate(((out_flags,), "out_flags", FLAG_TYPES, None))

    def forward(self, A, x, y, out_flags=None, stream=None):
        self._out_sizes(y, out_flags)
        a, xv, yv = self._arrays(A, x, y)
        _check(self._lib.gemv_ar_forward(self._h, a, xv, yv, _addr(out_flags), _stream(stream)))

    def unfused_forward(self, A, x, y, out_flags=None, stream=None):
        self._out_sizes(y, out_flags)
        a, xv, yv = self._arrays(A, x, y)
        _check(self._lib.gemv_ar_unfused_forward(self._h, a, xv, yv, _addr(out_flags), _stream(stream)))

    def status(self):
        """(timed_out, first missing peer flag); synchronises the device."""
        s = (ctypes.c_int32 * 2)()
        rc = self._lib.gemv_ar_status(self._h, s)
        if rc not in (EBAG_OK, EBAG_ETIMEOUT):
            _check(rc)
        return s[0], s[1]

    def reset(self):
        _check(self._lib.gemv_ar_reset(self._h))

    def launch_info(self):
        """(workgroups per rank P, threads per workgroup, tiles, resident workgroups, rows per tile)."""
        s = (ctypes.c_int32 * 5)()
        _check(self._lib.gemv_ar_launch_info(self._h, s))
        return tuple(s)

    def close(self):
        if getattr(self, "_h", None):
            self._lib.gemv_ar_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Q4Gemv:
    """A plan for products with 4-bit weights and group scales
    (``gemv_ar_q4_create``): `experts` matrices of M rows and K columns, a scale
    for every `group` columns, storage type dtype; glu=1: y = silu(gate) * up of
    the two halves of the M rows.  Methods mirror the C ABI and take torch tensors:
    codes uint8 [experts, M, ceil(K / 2)], scales [experts, M, ceil(K / group)],
    zeros uint8 of that shape or None, x and y with any step between rows, y of
    the plan's type or float32."""

    def __init__(self, M: int, K: int, group: int, dtype: int, experts: int = 1, glu: int = 0):
        lib = load()
        h = ctypes.c_void_p()
        _check(lib.gemv_ar_q4_create(ctypes.byref(h), int(M), int(K), int(group), int(dtype), int(experts), int(glu)))
        self._h = h
        self._lib = lib
        self._shape(M, K, group, dtype, experts, glu)

    def _shape(self, M, K, group, dtype, experts, glu):
        self.M, self.K, self.group, self.matrices = int(M), int(K), int(group), int(experts)
        self.wide = self.M // 2 if glu else self.M
        self.kind = {v: n for n, v in ROW_TYPES.items()}[int(dtype)]
        import torch
        self._u8, self._i32, self._f32, self._dtype = torch.uint8, torch.int32, torch.float32, getattr(torch, self.kind)
        rows = self.matrices * self.M
        self._all, self._codes, self._groups = rows * self.K, rows * ((self.K + 1) // 2), rows * -(-self.K // self.group)

    def _weights(self, codes, scales, zeros):
        if not (_fit(codes, self._u8, self._codes) and _fit(scales, self._dtype, self._groups) and
                (zeros is None or _fit(zeros, self._u8, self._groups))):
            _refuse((codes, "codes", ("uint8",), self._codes),
                    (scales, "scales", (self.kind,), self._groups * self._dtype.itemsize),
                    (zeros, "zeros", ("uint8",), self._groups))

    def quantize(self, w, codes, scales, zeros=None, stream=None):
        self._weights(codes, scales, zeros)
        if not _fit(w, self._dtype, self._all):
            _refuse((w, "w", (self.kind,), self._all * self._dtype.itemsize))
        _check(self._lib.gemv_ar_q4_quantize(self._h, w.data_ptr(), codes.data_ptr(), scales.data_ptr(), _addr(zeros),
                                             _stream(stream)))

    def _y(self, y, rows):
        kind = self.kind if y.dtype is self._dtype or y.dtype is not self._f32 else "float32"
        py, ldy, _ = _matrix(y, rows, self.wide, kind, "y")
        return py, ldy, ROW_TYPES[kind]

    def forward(self, codes, scales, zeros, x, y, stream=None):
        self._weights(codes, scales, zeros)
        rows = x.shape[0]
        px, ldx, _ = _matrix(x, rows, self.K, self.kind, "x")
        py, ldy, y_type = self._y(y, rows)
        _check(self._lib.gemv_ar_q4_forward(self._h, codes.data_ptr(), scales.data_ptr(), _addr(zeros), px, ldx, rows,
                                            py, ldy, y_type, _stream(stream)))

    def experts(self, codes, scales, zeros, x, offsets, y, src=None, k=1, stream=None):
        """gemv_ar_q4_experts; k: choices of a token, which src counts in."""
        self._weights(codes, scales, zeros)
        if not (_fit(offsets, self._i32, self.matrices + 1) and (src is None or _fit(src, self._i32, 0))):
            _refuse((offsets, "offsets", I32, 4 * (self.matrices + 1)), (src, "src", I32, 0))
        x_rows = x.shape[0]
        rows = x_rows if src is None else src.numel()
        px, ldx, _ = _matrix(x, x_rows, self.K, self.kind, "x")
        py, ldy, y_type = self._y(y, rows)
        _check(self._lib.gemv_ar_q4_experts(self._h, codes.data_ptr(), scales.data_ptr(), _addr(zeros), px, ldx, x_rows,
                                            offsets.data_ptr(), _addr(src), int(k), rows, py, ldy, y_type,
                                            _stream(stream)))

    def close(self):
        if getattr(self, "_h", None):
            self._lib.gemv_ar_q4_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Q8Gemv:
    """A plan for products in 8-bit integers with a scale for each token and each
    channel (``gemv_ar_q8_create``): `experts` matrices of M rows and K columns,
    x of dtype; glu=1: y = silu(gate) * up of the two halves of the M rows.
    Methods mirror the C ABI and take torch tensors: codes int8 [experts, M,
    pitch], scales float32 [experts, M], xq int8 [rows, pitch] and xs float32
    [rows], x and y with any step between rows, y of the plan's type or float32."""

    def __init__(self, M: int, K: int, dtype: int, experts: int = 1, glu: int = 0):
        lib = load()
        h = ctypes.c_void_p()
        _check(lib.gemv_ar_q8_create(ctypes.byref(h), int(M), int(K), int(dtype), int(experts), int(glu)))
        self._h = h
        self._lib = lib
        self._shape(M, K, dtype, experts, glu)

    def _shape(self, M, K, dtype, experts, glu):
        self.M, self.K, self.matrices = int(M), int(K), int(experts)
        self.pitch = -(-self.K // 128) * 128  # gemv_ar_q8_pitch
        self.wide = self.M // 2 if glu else self.M
        self.kind = {v: n for n, v in ROW_TYPES.items()}[int(dtype)]
        import torch
        self._i8, self._i32, self._f32, self._dtype = torch.int8, torch.int32, torch.float32, getattr(torch, self.kind)
        self._rows = self.matrices * self.M

    def _weights(self, codes, scales):
        if not (_fit(codes, self._i8, self._rows * self.pitch) and _fit(scales, self._f32, self._rows)):
            _refuse((codes, "codes", ("int8",), self._rows * self.pitch), (scales, "scales", F32, 4 * self._rows))

    def _x(self, x, xq, xs, rows):
        """(address, row step) of x, or of none; checks the rows' memory in 8 bits."""
        if not (_fit(xq, self._i8, rows * self.pitch) and _fit(xs, self._f32, rows)):
            _refuse((xq, "xq", ("int8",), rows * self.pitch), (xs, "xs", F32, 4 * rows))
        if x is None:
            return None, self.K
        px, ldx, _ = _matrix(x, rows, self.K, self.kind, "x")
        return px, ldx

    def _y(self, y, rows):
        kind = self.kind if y.dtype is self._dtype or y.dtype is not self._f32 else "float32"
        py, ldy, _ = _matrix(y, rows, self.wide, kind, "y")
        return py, ldy, ROW_TYPES[kind]

    def quantize(self, w, codes, scales, stream=None):
        self._weights(codes, scales)
        if not _fit(w, self._dtype, self._rows * self.K):
            _refuse((w, "w", (self.kind,), self._rows * self.K * self._dtype.itemsize))
        _check(self._lib.gemv_ar_q8_quantize(self._h, w.data_ptr(), codes.data_ptr(), scales.data_ptr(), _stream(stream)))

    def round(self, x, xq, xs, stream=None):
        rows = x.shape[0]
        px, ldx = self._x(x, xq, xs, rows)
        _check(self._lib.gemv_ar_q8_round(self._h, px, ldx, rows, xq.data_ptr(), xs.data_ptr(), _stream(stream)))

    def forward(self, codes, scales, x, y, xq, xs, stream=None):
        """gemv_ar_q8_forward; x None: the rows are those that round() left in xq and xs, as many as y has."""
        self._weights(codes, scales)
        rows = y.shape[0] if x is None else x.shape[0]
        px, ldx = self._x(x, xq, xs, rows)
        py, ldy, y_type = self._y(y, rows)
        _check(self._lib.gemv_ar_q8_forward(self._h, codes.data_ptr(), scales.data_ptr(), px, ldx, rows, xq.data_ptr(),
                                            xs.data_ptr(), py, ldy, y_type, _stream(stream)))

    def experts(self, codes, scales, x, offsets, y, xq, xs, src=None, k=1, stream=None):
        """gemv_ar_q8_experts; k: choices of a token, which src counts in; x None: the rows are xq's and xs's."""
        self._weights(codes, scales)
        if not (_fit(offsets, self._i32, self.matrices + 1) and (src is None or _fit(src, self._i32, 0))):
            _refuse((offsets, "offsets", I32, 4 * (self.matrices + 1)), (src, "src", I32, 0))
        x_rows = xs.numel() if x is None else x.shape[0]
        rows = x_rows if src is None else src.numel()
        px, ldx = self._x(x, xq, xs, x_rows)
        py, ldy, y_type = self._y(y, rows)
        _check(self._lib.gemv_ar_q8_experts(self._h, codes.data_ptr(), scales.data_ptr(), px, ldx, x_rows, xq.data_ptr(),
                                            xs.data_ptr(), offsets.data_ptr(), _addr(src), int(k), rows, py, ldy, y_type,
                                            _stream(stream)))

    def close(self):
        if getattr(self, "_h", None):
            self._lib.gemv_ar_q8_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
