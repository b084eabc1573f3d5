"""Thin ctypes binding over the C-ABI library (include/lasp.h).

Argument marshalling only: every step of the path runs in the HIP kernels.
PyTorch supplies device memory and the current stream. If the shared library
has not been built, importing this module raises: there is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblasp.so")

LASP_F32, LASP_BF16 = 0, 1
STATUS_NAMES = {0: "LASP_OK", 1: "LASP_ERR_NULL", 2: "LASP_ERR_SHAPE", 3: "LASP_ERR_DTYPE", 4: "LASP_ERR_DECAY",
                5: "LASP_ERR_WORKSPACE", 6: "LASP_ERR_ALIAS", 7: "LASP_ERR_HIP", 8: "LASP_ERR_ALIGN"}


class Shape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("N", ctypes.c_int32), ("D", ctypes.c_int32),
                ("chunk", ctypes.c_int32), ("dtype", ctypes.c_int32), ("segments", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("Dv", ctypes.c_int32)]


class RecShape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("N", ctypes.c_int32), ("D", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("coupled", ctypes.c_int32), ("ld", ctypes.c_int32)]


class RowsShape(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("C", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class GateShape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("N", ctypes.c_int32), ("D", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("gate", ctypes.c_int32), ("over", ctypes.c_int32), ("ld", ctypes.c_int32)]


class DeltaShape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("N", ctypes.c_int32), ("D", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("Dv", ctypes.c_int32), ("key_heads", ctypes.c_int32)]


class QkShape(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32) for name in ("B", "N", "H", "key_heads", "D", "dtype", "norm", "rot", "layout", "ld")]


class LaspError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)} ({status_str(status)})")


if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it first (python -c 'import __graft_entry__ as g; g.build()'). "
                      "There is no fallback path.")

_vp, _sz = ctypes.c_void_p, ctypes.c_size_t
_sp = ctypes.POINTER(Shape)


def _bind(handle):
    """Declare the C signatures of include/lasp.h on a loaded library."""
    handle.lasp_version.restype = ctypes.c_int
    handle.lasp_status_str.restype = ctypes.c_char_p
    handle.lasp_status_str.argtypes = [ctypes.c_int]
    handle.lasp_check_shape.argtypes = [_sp]
    handle.lasp_check_decay.argtypes = [ctypes.POINTER(ctypes.c_float), ctypes.c_int32]
    handle.lasp_tile_tokens.argtypes = [_sp]
    handle.lasp_tile_tokens.restype = ctypes.c_int32
    handle.lasp_num_segments.argtypes = [_sp]
    handle.lasp_num_segments.restype = ctypes.c_int32
    handle.lasp_state_cache_bytes.argtypes = [_sp]
    handle.lasp_state_cache_bytes.restype = _sz
    handle.lasp_scratch_bytes.argtypes = [_sp]
    handle.lasp_scratch_bytes.restype = _sz
    handle.lasp_fwd.argtypes = [_sp] + [_vp] * 9 + [_sz, _vp]
    handle.lasp_fwd.restype = ctypes.c_int
    handle.lasp_fwd_noalloc.argtypes = [_sp] + [_vp] * 9
    handle.lasp_fwd_noalloc.restype = ctypes.c_int
    handle.lasp_noalloc_scratch_limit.argtypes = []
    handle.lasp_noalloc_scratch_limit.restype = _sz
    handle.lasp_bwd.argtypes = [_sp] + [_vp] * 13 + [_sz, _vp]
    handle.lasp_bwd_recompute_scratch_bytes.argtypes = [_sp]
    handle.lasp_bwd_recompute_scratch_bytes.restype = _sz
    handle.lasp_gated_bwd_recompute_scratch_bytes.argtypes = [_sp]
    handle.lasp_gated_bwd_recompute_scratch_bytes.restype = _sz
    handle.lasp_bwd.restype = ctypes.c_int
    handle.lasp_check_log_decay.argtypes = [ctypes.POINTER(ctypes.c_float), ctypes.c_int64]
    handle.lasp_gated_state_cache_bytes.argtypes = [_sp]
    handle.lasp_gated_state_cache_bytes.restype = _sz
    handle.lasp_gated_scratch_bytes.argtypes = [_sp]
    handle.lasp_gated_scratch_bytes.restype = _sz
    handle.lasp_gated_fwd.argtypes = [_sp] + [_vp] * 9 + [_sz, _vp]
    handle.lasp_gated_fwd.restype = ctypes.c_int
    handle.lasp_gated_bwd.argtypes = [_sp] + [_vp] * 15 + [_sz, _vp]
    handle.lasp_gated_bwd.restype = ctypes.c_int
    handle.lasp_fwd_norm.argtypes = [_sp] + [_vp] * 5 + [ctypes.c_float] + [_vp] * 5 + [_sz, _vp]
    handle.lasp_fwd_norm.restype = ctypes.c_int
    handle.lasp_bwd_norm.argtypes = [_sp] + [_vp] * 15 + [_sz, _vp]
    handle.lasp_bwd_norm.restype = ctypes.c_int
    handle.lasp_gated_fwd_norm.argtypes = [_sp] + [_vp] * 5 + [ctypes.c_float] + [_vp] * 5 + [_sz, _vp]
    handle.lasp_gated_fwd_norm.restype = ctypes.c_int
    handle.lasp_gated_bwd_norm.argtypes = [_sp] + [_vp] * 17 + [_sz, _vp]
    handle.lasp_gated_bwd_norm.restype = ctypes.c_int
    handle.lasp_seq_scratch_bytes.argtypes = [_sp] + [ctypes.c_int32] * 3
    handle.lasp_seq_scratch_bytes.restype = _sz
    handle.lasp_seq_fwd.argtypes = [_sp, ctypes.c_int32] + [_vp] * 5 + [ctypes.c_int32, ctypes.c_float] + [_vp] * 5 + [_sz, _vp]
    handle.lasp_seq_fwd.restype = ctypes.c_int
    handle.lasp_seq_bwd.argtypes = [_sp, ctypes.c_int32] + [_vp] * 9 + [ctypes.c_int32] + [_vp] * 7 + [_sz, _vp]
    handle.lasp_seq_bwd.restype = ctypes.c_int
    handle.lasp_bidir_scratch_bytes.argtypes = [_sp]
    handle.lasp_bidir_scratch_bytes.restype = _sz
    handle.lasp_bidir_state.argtypes = [_sp, _vp, _vp, _vp, ctypes.c_int32, _vp, _sz, _vp]
    handle.lasp_bidir_state.restype = ctypes.c_int
    handle.lasp_bidir_fwd.argtypes = [_sp] + [_vp] * 4
    handle.lasp_bidir_fwd.restype = ctypes.c_int
    handle.lasp_bidir_bwd.argtypes = [_sp] + [_vp] * 9
    handle.lasp_bidir_bwd.restype = ctypes.c_int
    handle.lasp_profile_begin.argtypes = [ctypes.c_int32]
    handle.lasp_profile_end.argtypes = [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int32),
                                        ctypes.POINTER(ctypes.c_int32)]
    return handle


def _bind_bidir_sequence(handle):
    """The same for the calls of whole bidirectional sequences."""
    handle.lasp_bidir_seq_scratch_bytes.argtypes = [_sp, ctypes.c_int32]
    handle.lasp_bidir_seq_scratch_bytes.restype = _sz
    handle.lasp_bidir_seq_fwd.argtypes = [_sp, ctypes.c_int32] + [_vp] * 6 + [_sz, _vp]
    handle.lasp_bidir_seq_fwd.restype = ctypes.c_int
    handle.lasp_bidir_seq_bwd.argtypes = [_sp, ctypes.c_int32] + [_vp] * 10 + [_sz, _vp]
    handle.lasp_bidir_seq_bwd.restype = ctypes.c_int
    return handle


def _bind_blocks(handle):
    """The same for the gated recurrence and the norms around a mixer."""
    rec, rows, gate, f = ctypes.POINTER(RecShape), ctypes.POINTER(RowsShape), ctypes.POINTER(GateShape), ctypes.c_float
    for name, shape in (("rec", rec), ("addnorm", rows), ("gatenorm", gate)):
        size = getattr(handle, f"lasp_{name}_scratch_bytes")
        size.argtypes, size.restype = [shape], _sz
    handle.lasp_check_rec.argtypes, handle.lasp_check_rows.argtypes, handle.lasp_check_gate.argtypes = [rec], [rows], [gate]
    handle.lasp_rec_fwd.argtypes = [rec] + [_vp] * 7 + [_sz, _vp]
    handle.lasp_rec_bwd.argtypes = [rec] + [_vp] * 11 + [_sz, _vp]
    handle.lasp_addnorm_fwd.argtypes = [rows] + [_vp] * 4 + [f] + [_vp] * 3
    handle.lasp_addnorm_bwd.argtypes = [rows] + [_vp] * 4 + [f] + [_vp] * 7 + [_sz, _vp]
    handle.lasp_gatenorm_fwd.argtypes = [gate] + [_vp] * 3 + [f] + [_vp] * 2
    handle.lasp_gatenorm_bwd.argtypes = [gate] + [_vp] * 3 + [f] + [_vp] * 5 + [_sz, _vp]
    return handle


def _bind_delta(handle):
    """The same for the gated delta rule."""
    delta = ctypes.POINTER(DeltaShape)
    for name in ("cache", "scratch", "bwd_scratch"):
        size = getattr(handle, f"lasp_delta_{name}_bytes")
        size.argtypes, size.restype = [delta], _sz
    handle.lasp_check_delta.argtypes = [delta]
    handle.lasp_delta_fwd.argtypes = [delta] + [_vp] * 11 + [_sz, _vp]
    handle.lasp_delta_bwd.argtypes = [delta] + [_vp] * 16 + [_sz, _vp]
    return handle


def _bind_qk(handle):
    """The same for norms and rotation of queries and keys."""
    qk, f, d = ctypes.POINTER(QkShape), ctypes.c_float, ctypes.c_double
    handle.lasp_check_qk.argtypes = handle.lasp_qk_scratch_bytes.argtypes = [qk]
    handle.lasp_qk_scratch_bytes.restype = _sz
    handle.lasp_qk_fwd.argtypes = [qk] + [_vp] * 4 + [f] + [_vp] * 2 + [f] + [_vp] * 3
    handle.lasp_qk_bwd.argtypes = [qk] + [_vp] * 4 + [f] + [_vp] * 2 + [f] + [_vp] * 7 + [_sz, _vp]
    handle.lasp_rope_frequencies.argtypes = [ctypes.c_int32, d, ctypes.c_int32] + [d] * 4 + [_vp]
    return handle


lib = _bind_qk(_bind_delta(_bind_blocks(_bind_bidir_sequence(_bind(ctypes.CDLL(LIB_PATH))))))


def profile_begin(max_calls: int) -> None:
    rc = lib.lasp_profile_begin(int(max_calls))
    if rc != 0:
        raise LaspError(rc, "lasp_profile_begin")


def profile_end():
    """Returns ({'fwd': (local, scan, walk), 'bwd': (...)} summed milliseconds, fwd_calls, bwd_calls)."""
    ms = (ctypes.c_double * 6)()
    nf, nb = ctypes.c_int32(0), ctypes.c_int32(0)
    rc = lib.lasp_profile_end(ms, ctypes.byref(nf), ctypes.byref(nb))
    if rc != 0:
        raise LaspError(rc, "lasp_profile_end")
    return {"fwd": tuple(ms[0:3]), "bwd": tuple(ms[3:6])}, nf.value, nb.value


def status_str(status: int) -> str:
    return lib.lasp_status_str(int(status)).decode()


def version() -> int:
    return int(lib.lasp_version())


def make_shape(B, H, N, D, chunk, dtype, segments=0, kv_heads=0, Dv=0) -> Shape:
    if isinstance(dtype, torch.dtype):
        dtype = {torch.float32: LASP_F32, torch.bfloat16: LASP_BF16}.get(dtype, -1)
    elif isinstance(dtype, str):
        dtype = {"f32": LASP_F32, "bf16": LASP_BF16}.get(dtype, -1)
    return Shape(int(B), int(H), int(N), int(D), int(chunk), int(dtype), int(segments), int(kv_heads), int(Dv))


def check_shape(shape: Shape) -> int:
    return int(lib.lasp_check_shape(ctypes.byref(shape)))


def check_decay(decay_host) -> int:
    arr = (ctypes.c_float * len(decay_host))(*[float(x) for x in decay_host])
    return int(lib.lasp_check_decay(arr, len(decay_host)))


def tile_tokens(shape: Shape) -> int:
    return int(lib.lasp_tile_tokens(ctypes.byref(shape)))


def num_segments(shape: Shape) -> int:
    return int(lib.lasp_num_segments(ctypes.byref(shape)))


def state_cache_bytes(shape: Shape) -> int:
    return int(lib.lasp_state_cache_bytes(ctypes.byref(shape)))


def scratch_bytes(shape: Shape) -> int:
    return int(lib.lasp_scratch_bytes(ctypes.byref(shape)))


def _ptr(t: Optional[torch.Tensor]):
    """The address as a plain int, which the declared argument types take as it is: one new token for 8 x 16 heads 6.4 -> 5.9 us
    (the kernel alone 4.7) against a c_void_p for every one."""
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors handed to the library must be contiguous")
    return t.data_ptr()


def _stream(stream):
    if stream is None:   # the raw handle: building a Stream object takes 2.7 us of a 9 us call
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream


def lasp_fwd(shape: Shape, q, k, v, kv_in, decay, out, kv_out, state_cache, scratch, stream=None) -> None:
    """Enqueue the forward pass; raises LaspError on a non-zero status."""
    nbytes = scratch.numel() * scratch.element_size() if scratch is not None else 0
    rc = lib.lasp_fwd(ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(kv_in), _ptr(decay), _ptr(out),
                      _ptr(kv_out), _ptr(state_cache), _ptr(scratch), nbytes, _stream(stream))
    if rc != 0:
        raise LaspError(rc, "lasp_fwd")


def noalloc_scratch_limit() -> int:
    return int(lib.lasp_noalloc_scratch_limit())


def lasp_fwd_noalloc(shape: Shape, q, k, v, kv_in, decay, out, kv_out, state_cache, stream=None) -> None:
    """lasp_fwd with the library's own fixed scratch (no workspace argument); raises LaspError on a non-zero status."""
    rc = lib.lasp_fwd_noalloc(ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(kv_in), _ptr(decay), _ptr(out),
                              _ptr(kv_out), _ptr(state_cache), _stream(stream))
    if rc != 0:
        raise LaspError(rc, "lasp_fwd_noalloc")


def bwd_recompute_scratch_bytes(shape: Shape) -> int:
    return int(lib.lasp_bwd_recompute_scratch_bytes(ctypes.byref(shape)))


def gated_bwd_recompute_scratch_bytes(shape: Shape) -> int:
    return int(lib.lasp_gated_bwd_recompute_scratch_bytes(ctypes.byref(shape)))


def lasp_bwd(shape: Shape, q, k, v, dout, kv_in, dkv_out, decay, state_cache, dq, dk, dv, dkv_in, scratch,
             stream=None) -> None:
    """Enqueue the backward pass (state_cache None = the states are rebuilt from k, v, kv_in); raises LaspError
    on a non-zero status."""
    nbytes = scratch.numel() * scratch.element_size() if scratch is not None else 0
    rc = lib.lasp_bwd(ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(dout), _ptr(kv_in), _ptr(dkv_out), _ptr(decay),
                      _ptr(state_cache), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dkv_in), _ptr(scratch), nbytes,
                      _stream(stream))
    if rc != 0:
        raise LaspError(rc, "lasp_bwd")


def check_log_decay(log_g_host) -> int:
    import numpy as np
    a = np.ascontiguousarray(log_g_host, dtype=np.float32).ravel()
    return int(lib.lasp_check_log_decay(a.ctypes.data_as(ctypes.POINTER(ctypes.c_float)), a.size))


def gated_state_cache_bytes(shape: Shape) -> int:
    return int(lib.lasp_gated_state_cache_bytes(ctypes.byref(shape)))


def gated_scratch_bytes(shape: Shape) -> int:
    return int(lib.lasp_gated_scratch_bytes(ctypes.byref(shape)))


def lasp_gated_fwd(shape: Shape, q, k, v, log_g, kv_in, out, kv_out, state_cache, scratch, stream=None) -> None:
    """Forward with a decay per token (log_g: float32 [B,H,N]); raises LaspError on a non-zero status."""
    nbytes = scratch.numel() * scratch.element_size() if scratch is not None else 0
    rc = lib.lasp_gated_fwd(ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(log_g), _ptr(kv_in), _ptr(out),
                            _ptr(kv_out), _ptr(state_cache), _ptr(scratch), nbytes, _stream(stream))
    if rc != 0:
        raise LaspError(rc, "lasp_gated_fwd")


def lasp_gated_bwd(shape: Shape, q, k, v, dout, log_g, kv_in, kv_out, dkv_out, state_cache, dq, dk, dv, dlog_g, dkv_in,
                   scratch, stream=None) -> None:
    """Backward with a decay per token; raises LaspError on a non-zero status."""
    nbytes = scratch.numel() * scratch.element_size() if scratch is not None else 0
    rc = lib.lasp_gated_bwd(ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(dout), _ptr(log_g), _ptr(kv_in), _ptr(kv_out),
                            _ptr(dkv_out), _ptr(state_cache), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dlog_g),
                            _ptr(dkv_in), _ptr(scratch), nbytes, _stream(stream))
    if rc != 0:
        raise LaspError(rc, "lasp_gated_bwd")


def lasp_fwd_norm(shape: Shape, q, k, v, kv_in, decay, eps, out, rstd, kv_out, state_cache, scratch,
                  stream=None) -> None:
    """Forward with the normalised output (out = Norm(o), rstd: float32 [B,H,N]); raises LaspError."""
    nbytes = scratch.numel() * scratch.element_size() if scratch is not None else 0
    rc = lib.lasp_fwd_norm(ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(kv_in), _ptr(decay), float(eps),
                           _ptr(out), _ptr(rstd), _ptr(kv_out), _ptr(state_cache), _ptr(scratch), nbytes,
                           _stream(stream))
    if rc != 0:
        raise LaspError(rc, "lasp_fwd_norm")


def lasp_bwd_norm(shape: Shape, q, k, v, out, rstd, dout, kv_in, dkv_out, decay, state_cache, dq, dk, dv, dkv_in,
                  scratch, stream=None) -> None:
    """Backward of lasp_fwd_norm (dout: gradient w.r.t. the normalised output); raises LaspError."""
    nbytes = scratch.numel() * scratch.element_size() if scratch is not None else 0
    rc = lib.lasp_bwd_norm(ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(rstd), _ptr(dout),
                           _ptr(kv_in), _ptr(dkv_out), _ptr(decay), _ptr(state_cache), _ptr(dq), _ptr(dk), _ptr(dv),
                           _ptr(dkv_in), _ptr(scratch), nbytes, _stream(stream))
    if rc != 0:
        raise LaspError(rc, "lasp_bwd_norm")


def lasp_gated_fwd_norm(shape: Shape, q, k, v, log_g, kv_in, eps, out, rstd, kv_out, state_cache, scratch,
                        stream=None) -> None:
    """Per-token decay and normalised output together; raises LaspError on a non-zero status."""
    nbytes = scratch.numel() * scratch.element_size() if scratch is not None else 0
    rc = lib.lasp_gated_fwd_norm(ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(log_g), _ptr(kv_in), float(eps),
                                 _ptr(out), _ptr(rstd), _ptr(kv_out), _ptr(state_cache), _ptr(scratch), nbytes,
                                 _stream(stream))
    if rc != 0:
        raise LaspError(rc, "lasp_gated_fwd_norm")


def lasp_gated_bwd_norm(shape: Shape, q, k, v, out, rstd, dout, log_g, kv_in, kv_out, dkv_out, state_cache, dq, dk, dv,
                        dlog_g, dkv_in, scratch, stream=None) -> None:
    """Backward of lasp_gated_fwd_norm; raises LaspError on a non-zero status."""
    nbytes = scratch.numel() * scratch.element_size() if scratch is not None else 0
    rc = lib.lasp_gated_bwd_norm(ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(rstd), _ptr(dout),
                                 _ptr(log_g), _ptr(kv_in), _ptr(kv_out), _ptr(dkv_out), _ptr(state_cache), _ptr(dq), _ptr(dk),
                                 _ptr(dv), _ptr(dlog_g), _ptr(dkv_in), _ptr(scratch), nbytes, _stream(stream))
    if rc != 0:
        raise LaspError(rc, "lasp_gated_bwd_norm")


def seq_scratch_bytes(shape: Shape, T: int, token: bool, recompute: bool) -> int:
    return int(lib.lasp_seq_scratch_bytes(ctypes.byref(shape), int(T), int(token), int(recompute)))


def _tables(*lists):
    """Addresses of the first n tensors of every (list, n) in one host array: (the array, which the caller keeps until its
    call has returned, the address of each list's part of it; None for a list that is None)."""
    flat, first = [], []
    for tensors, n in lists:
        if tensors is None:
            first.append(None)
            continue
        first.append(8 * len(flat))
        for t in range(n):
            t = tensors[t]
            if t is None:
                flat.append(0)
            elif t.is_contiguous():
                flat.append(t.data_ptr())
            else:
                raise ValueError("tensors handed to the library must be contiguous")
    table = (ctypes.c_size_t * len(flat))(*flat)
    base = ctypes.addressof(table)
    return table, [None if n is None else base + n for n in first]


def lasp_seq_fwd(shape: Shape, T, q, k, v, kv_in, decay, token, eps, out, rstd, kv, state_cache, scratch, stream=None) -> None:
    """Enqueue the forward pass of T sub-sequences (lists of T tensors, kv of T + 1; decay: a tensor, or a list of T with
    `token`; rstd None = outputs not normalised); raises LaspError on a non-zero status."""
    keep, (q, k, v, decay, out, rstd, kv, state_cache) = _tables(
        (q, T), (k, T), (v, T), (decay, T) if token else ([decay], 1), (out, T), (rstd, T), (kv, T + 1), (state_cache, T))
    rc = lib.lasp_seq_fwd(ctypes.byref(shape), T, q, k, v, _ptr(kv_in), decay, token, eps, out, rstd, kv, state_cache, _ptr(scratch),
                          scratch.numel() * scratch.element_size(), _stream(stream))
    if rc != 0:
        raise LaspError(rc, "lasp_seq_fwd")


def lasp_seq_bwd(shape: Shape, T, q, k, v, out, rstd, dout, kv, dkv_out, decay, token, state_cache, dq, dk, dv, dlog_g, dkv, scratch,
                 stream=None) -> None:
    """Enqueue the backward pass of T sub-sequences; raises LaspError on a non-zero status."""
    keep, (q, k, v, out, rstd, dout, kv, decay, state_cache, dq, dk, dv, dlog_g, dkv) = _tables(
        (q, T), (k, T), (v, T), (out, T), (rstd, T), (dout, T), (kv, T + 1), (decay, T) if token else ([decay], 1), (state_cache, T),
        (dq, T), (dk, T), (dv, T), (dlog_g, T), (dkv, T + 1))
    rc = lib.lasp_seq_bwd(ctypes.byref(shape), T, q, k, v, out, rstd, dout, kv, _ptr(dkv_out), decay, token, state_cache, dq, dk, dv,
                          dlog_g, dkv, _ptr(scratch), scratch.numel() * scratch.element_size(), _stream(stream))
    if rc != 0:
        raise LaspError(rc, "lasp_seq_bwd")


def bidir_scratch_bytes(shape: Shape) -> int:
    return int(lib.lasp_bidir_scratch_bytes(ctypes.byref(shape)))


def lasp_bidir_state(shape: Shape, x, y, state, accumulate, scratch, stream=None) -> None:
    """state (+)= sum over tokens of x_s y_s^T (bidirectional attention); raises LaspError on a non-zero status."""
    nbytes = scratch.numel() * scratch.element_size() if scratch is not None else 0
    rc = lib.lasp_bidir_state(ctypes.byref(shape), _ptr(x), _ptr(y), _ptr(state), int(bool(accumulate)), _ptr(scratch),
                              nbytes, _stream(stream))
    if rc != 0:
        raise LaspError(rc, "lasp_bidir_state")


def lasp_bidir_fwd(shape: Shape, q, kv, out, stream=None) -> None:
    """out = q kv; raises LaspError on a non-zero status."""
    rc = lib.lasp_bidir_fwd(ctypes.byref(shape), _ptr(q), _ptr(kv), _ptr(out), _stream(stream))
    if rc != 0:
        raise LaspError(rc, "lasp_bidir_fwd")


def lasp_bidir_bwd(shape: Shape, k, v, dout, kv, dkv, dq, dk, dv, stream=None) -> None:
    """dq = dout kv^T, dk = v dkv^T, dv = k dkv; raises LaspError on a non-zero status."""
    rc = lib.lasp_bidir_bwd(ctypes.byref(shape), _ptr(k), _ptr(v), _ptr(dout), _ptr(kv), _ptr(dkv), _ptr(dq), _ptr(dk),
                            _ptr(dv), _stream(stream))
    if rc != 0:
        raise LaspError(rc, "lasp_bidir_bwd")


def bidir_seq_scratch_bytes(shapes, T) -> int:
    return int(lib.lasp_bidir_seq_scratch_bytes(shapes, T))


def lasp_bidir_seq_fwd(shapes, T, q, k, v, kv, out, scratch, stream=None) -> None:
    """kv = sum over T sub-sequences (shapes: a ctypes array of T, lists of T tensors) of k^T v, every out = q kv; raises
    LaspError on a non-zero status."""
    keep, (q, k, v, out) = _tables((q, T), (k, T), (v, T), (out, T))
    rc = lib.lasp_bidir_seq_fwd(shapes, T, q, k, v, _ptr(kv), out, _ptr(scratch), scratch.numel() * scratch.element_size(), _stream(stream))
    if rc != 0:
        raise LaspError(rc, "lasp_bidir_seq_fwd")


def lasp_bidir_seq_bwd(shapes, T, q, k, v, dout, kv, dkv, dq, dk, dv, scratch, stream=None) -> None:
    """dkv = sum over T sub-sequences of q^T dout, and every dq, dk, dv; raises LaspError on a non-zero status."""
    keep, (q, k, v, dout, dq, dk, dv) = _tables((q, T), (k, T), (v, T), (dout, T), (dq, T), (dk, T), (dv, T))
    rc = lib.lasp_bidir_seq_bwd(shapes, T, q, k, v, dout, _ptr(kv), _ptr(dkv), dq, dk, dv, _ptr(scratch),
                                scratch.numel() * scratch.element_size(), _stream(stream))
    if rc != 0:
        raise LaspError(rc, "lasp_bidir_seq_bwd")


# ---- The gated recurrence and the norms around a mixer --------------------------
GATES = {"none": 0, "identity": 1, "sigmoid": 2, "silu": 3}
OVER = {"head": 0, "token": 1}
_TORCH = {LASP_F32: torch.float32, LASP_BF16: torch.bfloat16}


def _dtype_code(dtype):
    if isinstance(dtype, torch.dtype):
        return {torch.float32: LASP_F32, torch.bfloat16: LASP_BF16}.get(dtype, -1)
    return {"f32": LASP_F32, "bf16": LASP_BF16}.get(dtype, -1) if isinstance(dtype, str) else int(dtype)


def make_rec_shape(B, N, D, dtype, coupled=False, ld=0) -> RecShape:
    return RecShape(int(B), int(N), int(D), _dtype_code(dtype), int(bool(coupled)), int(ld))


def make_rows(rows, C, dtype) -> RowsShape:
    return RowsShape(int(rows), int(C), _dtype_code(dtype))


def make_gate_shape(B, H, N, D, dtype, gate="silu", over="head", ld=0) -> GateShape:
    """gate: one of GATES, over: one of OVER (unknown names are refused by the calls)."""
    return GateShape(int(B), int(H), int(N), int(D), _dtype_code(dtype), GATES.get(gate, -1), OVER.get(over, -1), int(ld))


def check_rec(shape: RecShape) -> int:
    return int(lib.lasp_check_rec(ctypes.byref(shape)))


def check_rows(shape: RowsShape) -> int:
    return int(lib.lasp_check_rows(ctypes.byref(shape)))


def check_gate(shape: GateShape) -> int:
    return int(lib.lasp_check_gate(ctypes.byref(shape)))


def rec_scratch_bytes(shape: RecShape) -> int:
    return int(lib.lasp_rec_scratch_bytes(ctypes.byref(shape)))


def addnorm_scratch_bytes(shape: RowsShape) -> int:
    return int(lib.lasp_addnorm_scratch_bytes(ctypes.byref(shape)))


def gatenorm_scratch_bytes(shape: GateShape) -> int:
    return int(lib.lasp_gatenorm_scratch_bytes(ctypes.byref(shape)))


def _refuse(t, name, numel, dtype, at):
    if t.get_device() < 0:
        raise ValueError(f"{name}: must be on a GPU")
    if t.get_device() != at:
        raise ValueError(f"{name}: on device {t.get_device()}, other tensors of the call on {at}")
    raise ValueError(f"{name}: must be contiguous, {numel} elements of {dtype}, not {tuple(t.shape)} of {t.dtype}")


def _addr(t, name, numel, dtype, at):
    """The address of a contiguous tensor of `numel` elements on device `at` (None passes). These calls take no sizes but the
    plan's: a tensor of another one would be read past its end. (Five look-ups, 0.6 us.)"""
    if t is None:
        return None
    if t.numel() != numel or t.dtype is not dtype or t.get_device() != at or at < 0 or not t.is_contiguous():
        _refuse(t, name, numel, dtype, at)
    return t.data_ptr()


def _addr_rows(t, name, B, N, width, ld, dtype, at):
    """The same of [B][N] rows of `width` elements, `ld` from row to row (0 = width)."""
    if t is None or ld == 0 or ld == width:
        return _addr(t, name, B * N * width, dtype, at)
    if t.get_device() != at or at < 0 or t.dtype is not dtype:
        _refuse(t, name, B * N * width, dtype, at)
    if t.shape != (B, N, width) or (width > 1 and t.stride(2) != 1) or (N > 1 and t.stride(1) != ld) or (B > 1 and t.stride(0) != N * ld):
        raise ValueError(f"{name}: must be [{B}][{N}][{width}], rows {ld} apart, not {tuple(t.shape)} with strides {t.stride()}")
    return t.data_ptr()


def _room(t, at):
    """Address and size of a workspace."""
    if t is None:
        return None, 0
    if t.get_device() != at or at < 0 or not t.is_contiguous():
        _refuse(t, "scratch", t.numel(), t.dtype, at)
    return t.data_ptr(), t.numel() * t.element_size()


def _call(fn, where, at, stream, *args):
    """On `stream`, or the current one of the tensors' device."""
    if at == torch._C._cuda_getDevice():
        rc = fn(*args, torch._C._cuda_getCurrentRawStream(at) if stream is None else stream.cuda_stream)
    else:
        with torch.cuda.device(at):
            rc = fn(*args, torch._C._cuda_getCurrentRawStream(at) if stream is None else stream.cuda_stream)
    if rc != 0:
        raise LaspError(rc, where)


def _home(t, name, shape, check):
    """The data type and device of a call: those of the plan and of its first tensor."""
    dtype = _TORCH.get(shape.dtype)
    if dtype is None or t is None:
        raise LaspError(check(shape) or 1, name)
    return dtype, t.get_device()


def lasp_rec_fwd(shape: RecShape, x, log_a, h_in, lens, out, h_out, scratch, stream=None) -> None:
    """h_s = exp(log_a_s) h_{s-1} + b_s x_s per channel: x, log_a [B,N,D] (rows shape.ld apart), out [B,N,D], h_in, h_out float32
    [B,D] or None, lens int32 [B] or None; raises LaspError on a non-zero status."""
    (d, at), f, B, N, D, ld = _home(x, "lasp_rec_fwd", shape, check_rec), torch.float32, shape.B, shape.N, shape.D, shape.ld
    n = B * D
    _call(lib.lasp_rec_fwd, "lasp_rec_fwd", at, stream, ctypes.byref(shape), _addr_rows(x, "x", B, N, D, ld, d, at),
          _addr_rows(log_a, "log_a", B, N, D, ld, d, at), _addr(h_in, "h_in", n, f, at), _addr(lens, "lens", B, torch.int32, at),
          _addr(out, "out", N * n, d, at), _addr(h_out, "h_out", n, f, at), *_room(scratch, at))


def lasp_rec_bwd(shape: RecShape, x, log_a, out, h_in, lens, dout, dh_out, dx, dlog_a, dh_in, scratch, stream=None) -> None:
    """Gradients dx, dlog_a (as x, log_a), dh_in of lasp_rec_fwd, from its `out` (x: needed when coupled); raises LaspError on a
    non-zero status."""
    (d, at), f, B, N, D, ld = _home(log_a, "lasp_rec_bwd", shape, check_rec), torch.float32, shape.B, shape.N, shape.D, shape.ld
    n = B * D
    _call(lib.lasp_rec_bwd, "lasp_rec_bwd", at, stream, ctypes.byref(shape), _addr_rows(x, "x", B, N, D, ld, d, at),
          _addr_rows(log_a, "log_a", B, N, D, ld, d, at), _addr(out, "out", N * n, d, at), _addr(h_in, "h_in", n, f, at),
          _addr(lens, "lens", B, torch.int32, at), _addr(dout, "dout", N * n, d, at), _addr(dh_out, "dh_out", n, f, at),
          _addr_rows(dx, "dx", B, N, D, ld, d, at), _addr_rows(dlog_a, "dlog_a", B, N, D, ld, d, at), _addr(dh_in, "dh_in", n, f, at),
          *_room(scratch, at))


def lasp_addnorm_fwd(shape: RowsShape, r, x, scale, weight, eps, r_out, y, stream=None) -> None:
    """r_out = r + scale * x, y = weight * r_out / rms(r_out), rows of C (scale, weight float32 [C] or None; x, r_out None: the norm
    of r alone); raises LaspError on a non-zero status."""
    (d, at), f, C = _home(r, "lasp_addnorm_fwd", shape, check_rows), torch.float32, shape.C
    n = shape.rows * C
    _call(lib.lasp_addnorm_fwd, "lasp_addnorm_fwd", at, stream, ctypes.byref(shape), _addr(r, "r", n, d, at), _addr(x, "x", n, d, at),
          _addr(scale, "scale", C, f, at), _addr(weight, "weight", C, f, at), eps, _addr(r_out, "r_out", n, d, at), _addr(y, "y", n, d, at))


def lasp_addnorm_bwd(shape: RowsShape, r_out, x, scale, weight, eps, dy, dr_out, dr, dx, dweight, dscale, scratch, stream=None) -> None:
    """Gradients of lasp_addnorm_fwd from its r_out (dr_out: what reaches r_out past the norm, or None; dx, dweight, dscale may be
    None, scratch then too); raises LaspError on a non-zero status."""
    (d, at), f, C = _home(r_out, "lasp_addnorm_bwd", shape, check_rows), torch.float32, shape.C
    n = shape.rows * C
    _call(lib.lasp_addnorm_bwd, "lasp_addnorm_bwd", at, stream, ctypes.byref(shape), _addr(r_out, "r_out", n, d, at),
          _addr(x, "x", n, d, at), _addr(scale, "scale", C, f, at), _addr(weight, "weight", C, f, at), eps, _addr(dy, "dy", n, d, at),
          _addr(dr_out, "dr_out", n, d, at), _addr(dr, "dr", n, d, at), _addr(dx, "dx", n, d, at), _addr(dweight, "dweight", C, f, at),
          _addr(dscale, "dscale", C, f, at), *_room(scratch, at))


def lasp_gatenorm_fwd(shape: GateShape, o, u, weight, eps, y, stream=None) -> None:
    """y = weight * o / rms(o) * act(u): o [B,H,N,D], u [B,N,H*D] (rows shape.ld apart), y [B,N,H*D], weight float32 [H*D] or None;
    raises LaspError on a non-zero status."""
    (d, at), B, N, C = _home(o, "lasp_gatenorm_fwd", shape, check_gate), shape.B, shape.N, shape.H * shape.D
    n = B * N * C
    _call(lib.lasp_gatenorm_fwd, "lasp_gatenorm_fwd", at, stream, ctypes.byref(shape), _addr(o, "o", n, d, at),
          _addr_rows(u, "u", B, N, C, shape.ld, d, at), _addr(weight, "weight", C, torch.float32, at), eps, _addr(y, "y", n, d, at))


def lasp_gatenorm_bwd(shape: GateShape, o, u, weight, eps, dy, do, du, dweight, scratch, stream=None) -> None:
    """Gradients of lasp_gatenorm_fwd: do as o, du as u, dweight (may be None, scratch then too); raises LaspError on a non-zero
    status."""
    (d, at), f, B, N, C = _home(o, "lasp_gatenorm_bwd", shape, check_gate), torch.float32, shape.B, shape.N, shape.H * shape.D
    n = B * N * C
    _call(lib.lasp_gatenorm_bwd, "lasp_gatenorm_bwd", at, stream, ctypes.byref(shape), _addr(o, "o", n, d, at),
          _addr_rows(u, "u", B, N, C, shape.ld, d, at), _addr(weight, "weight", C, f, at), eps, _addr(dy, "dy", n, d, at),
          _addr(do, "do", n, d, at), _addr_rows(du, "du", B, N, C, shape.ld, d, at), _addr(dweight, "dweight", C, f, at),
          *_room(scratch, at))


# ---- Queries and keys: norm, rotation, heads first ----------------------------------
NORMS = {"none": 0, "rms": 1, "l2": 2}
ROTATIONS = {"half": 0, "interleaved": 1}
ROPES = {"none": 0, "linear": 1, "base": 2, "bands": 3}


def make_qk_shape(B, N, H, key_heads, D, dtype, norm="rms", rot=0, layout="half", ld=0) -> QkShape:
    """norm: one of NORMS, layout: one of ROTATIONS (unknown names are refused by the calls)."""
    return QkShape(int(B), int(N), int(H), int(key_heads), int(D), _dtype_code(dtype), NORMS.get(norm, -1), int(rot), ROTATIONS.get(layout, -1),
                   int(ld))


def check_qk(shape: QkShape) -> int:
    return int(lib.lasp_check_qk(ctypes.byref(shape)))


def qk_scratch_bytes(shape: QkShape) -> int:
    return int(lib.lasp_qk_scratch_bytes(ctypes.byref(shape)))


def rope_frequencies(rot, base=10000.0, scaling="none", factor=1.0, trained=4096.0, few_turns=1.0, many_turns=32.0, device="cuda") -> torch.Tensor:
    """float64 [rot/2], radians per position, for lasp_qk_fwd; scaling: one of ROPES, for a context `factor` times the `trained` one."""
    freq = torch.empty(max(int(rot), 0) // 2, dtype=torch.float64)
    rc = lib.lasp_rope_frequencies(int(rot), float(base), ROPES.get(scaling, -1), float(factor), float(trained), float(few_turns),
                                   float(many_turns), freq.data_ptr() or None)
    if rc != 0:
        raise LaspError(rc, "rope_frequencies")
    return freq.to(device)


def _qk_args(shape: QkShape, xq, xk, wq, wk, freq, pos, at, d):
    """Addresses of what both calls read."""
    B, N, D, f = shape.B, shape.N, shape.D, torch.float32
    keys = shape.key_heads > 0
    return (_addr_rows(xq, "xq", B, N, shape.H * D, shape.ld, d, at),
            _addr_rows(xk, "xk", B, N, shape.key_heads * D, shape.ld, d, at) if keys else None, _addr(wq, "wq", D, f, at),
            _addr(wk, "wk", D, f, at) if keys else None, _addr(freq, "freq", shape.rot // 2, torch.float64, at) if shape.rot else None,
            _addr(pos, "pos", B * N, torch.int32, at) if shape.rot else None)


def lasp_qk_fwd(shape: QkShape, xq, xk, wq, wk, eps, freq, pos, amplitude, q, k, stream=None) -> None:
    """Norm and rotation by head: xq [B,N,H*D], xk [B,N,key_heads*D] (rows shape.ld apart) to q [B,H,N,D], k [B,key_heads,N,D]; wq, wk float32
    [D] or None, freq float64 [rot/2] (rope_frequencies), pos int32 [B,N] or None; raises LaspError on a non-zero status."""
    (d, at), n = _home(xq, "lasp_qk_fwd", shape, check_qk), shape.B * shape.N * shape.D
    xq, xk, wq, wk, freq, pos = _qk_args(shape, xq, xk, wq, wk, freq, pos, at, d)
    _call(lib.lasp_qk_fwd, "lasp_qk_fwd", at, stream, ctypes.byref(shape), xq, xk, wq, wk, eps, freq, pos, amplitude,
          _addr(q, "q", n * shape.H, d, at), _addr(k, "k", n * shape.key_heads, d, at) if shape.key_heads else None)


def lasp_qk_bwd(shape: QkShape, xq, xk, wq, wk, eps, freq, pos, amplitude, dq, dk, dxq, dxk, dwq, dwk, scratch, stream=None) -> None:
    """Gradients dxq, dxk (as xq, xk), dwq, dwk (may be None, scratch then too) of lasp_qk_fwd; raises LaspError on a non-zero status."""
    (d, at), n, f = _home(dq, "lasp_qk_bwd", shape, check_qk), shape.B * shape.N * shape.D, torch.float32
    B, N, D, keys = shape.B, shape.N, shape.D, shape.key_heads > 0
    xq, xk, wq, wk, freq, pos = _qk_args(shape, xq, xk, wq, wk, freq, pos, at, d)
    _call(lib.lasp_qk_bwd, "lasp_qk_bwd", at, stream, ctypes.byref(shape), xq, xk, wq, wk, eps, freq, pos, amplitude,
          _addr(dq, "dq", n * shape.H, d, at), _addr(dk, "dk", n * shape.key_heads, d, at) if keys else None,
          _addr_rows(dxq, "dxq", B, N, shape.H * D, shape.ld, d, at),
          _addr_rows(dxk, "dxk", B, N, shape.key_heads * D, shape.ld, d, at) if keys else None, _addr(dwq, "dwq", D, f, at),
          _addr(dwk, "dwk", D, f, at) if keys else None, *_room(scratch, at))


# ---- The gated delta rule ---------------------------------------------------------
def make_delta_shape(B, H, N, D, dtype, Dv=0, key_heads=0) -> DeltaShape:
    return DeltaShape(int(B), int(H), int(N), int(D), _dtype_code(dtype), int(Dv), int(key_heads))


def check_delta(shape: DeltaShape) -> int:
    return int(lib.lasp_check_delta(ctypes.byref(shape)))


def delta_cache_bytes(shape: DeltaShape) -> int:
    return int(lib.lasp_delta_cache_bytes(ctypes.byref(shape)))


def delta_scratch_bytes(shape: DeltaShape) -> int:
    return int(lib.lasp_delta_scratch_bytes(ctypes.byref(shape)))


def delta_bwd_scratch_bytes(shape: DeltaShape) -> int:
    return int(lib.lasp_delta_bwd_scratch_bytes(ctypes.byref(shape)))


def _delta_numels(shape: DeltaShape):
    """Elements of q, of v, of a state and of beta."""
    tokens, Dv = shape.B * shape.N, shape.Dv or shape.D
    return (tokens * (shape.key_heads or shape.H) * shape.D, tokens * shape.H * Dv, shape.B * shape.H * shape.D * Dv, tokens * shape.H)


def _cache_addr(cache, shape, at):
    """The address of a state cache (None passes), which the library takes without its size."""
    addr, size = _room(cache, at)
    if addr is not None and size < delta_cache_bytes(shape):
        raise LaspError(5, "state_cache")
    return addr


def lasp_delta_fwd(shape: DeltaShape, q, k, v, log_g, beta, kv_in, lens, out, kv_out, state_cache, scratch, stream=None) -> None:
    """Gated delta rule: q, k [B,key_heads,N,D], v, out [B,H,N,Dv], log_g (or None), beta float32 [B,H,N], kv_in (or None), kv_out float32
    [B,H,D,Dv], lens int32 [B] or None, state_cache None when no backward pass follows; raises LaspError on a non-zero status."""
    (d, at), f = _home(q, "lasp_delta_fwd", shape, check_delta), torch.float32
    nq, nv, ns, ng = _delta_numels(shape)
    _call(lib.lasp_delta_fwd, "lasp_delta_fwd", at, stream, ctypes.byref(shape), _addr(q, "q", nq, d, at), _addr(k, "k", nq, d, at),
          _addr(v, "v", nv, d, at), _addr(log_g, "log_g", ng, f, at), _addr(beta, "beta", ng, f, at), _addr(kv_in, "kv_in", ns, f, at),
          _addr(lens, "lens", shape.B, torch.int32, at), _addr(out, "out", nv, d, at), _addr(kv_out, "kv_out", ns, f, at),
          _cache_addr(state_cache, shape, at) if state_cache is not None else None, *_room(scratch, at))


def lasp_delta_bwd(shape: DeltaShape, q, k, v, log_g, beta, lens, dout, dkv_out, state_cache, dq, dk, dv, dlog_g, dbeta, dkv_in, scratch,
                   stream=None) -> None:
    """Gradients of lasp_delta_fwd from the state_cache it filled (dkv_out may be None; dlog_g goes with log_g); raises LaspError on a
    non-zero status."""
    (d, at), f = _home(q, "lasp_delta_bwd", shape, check_delta), torch.float32
    nq, nv, ns, ng = _delta_numels(shape)
    _call(lib.lasp_delta_bwd, "lasp_delta_bwd", at, stream, ctypes.byref(shape), _addr(q, "q", nq, d, at), _addr(k, "k", nq, d, at),
          _addr(v, "v", nv, d, at), _addr(log_g, "log_g", ng, f, at), _addr(beta, "beta", ng, f, at),
          _addr(lens, "lens", shape.B, torch.int32, at), _addr(dout, "dout", nv, d, at), _addr(dkv_out, "dkv_out", ns, f, at),
          _cache_addr(state_cache, shape, at), _addr(dq, "dq", nq, d, at), _addr(dk, "dk", nq, d, at), _addr(dv, "dv", nv, d, at),
          _addr(dlog_g, "dlog_g", ng, f, at), _addr(dbeta, "dbeta", ng, f, at), _addr(dkv_in, "dkv_in", ns, f, at), *_room(scratch, at))


class Workspace:
    """Device buffers one (shape) needs besides the tensors: state cache and scratch."""

    def __init__(self, shape: Shape, device="cuda", with_cache=True):
        self.shape = shape
        if check_shape(shape) != 0:
            raise LaspError(check_shape(shape), "Workspace")
        self.cache = torch.empty(state_cache_bytes(shape), dtype=torch.uint8, device=device) if with_cache else None
        self.scratch = torch.empty(scratch_bytes(shape), dtype=torch.uint8, device=device)
