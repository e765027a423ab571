"""Thin ctypes binding over the C ABI declared in include/sbc.h.

Argument marshalling only: torch supplies device memory and the current CUDA
stream, every step of the method runs in the library's kernels.  The library
is loaded on first use; if it is missing or cannot be loaded the call raises
-- there is no other path.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import List, Optional, Sequence, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsbc_b200.so")

SBC_OK, SBC_EINVAL, SBC_ECAPACITY, SBC_ENONFINITE, SBC_ECORRUPT, SBC_ETIMEOUT, SBC_ECUDA = 0, -1, -2, -3, -4, -5, -6
STATUS_NONFINITE, STATUS_CORRUPT, STATUS_RANGE, STATUS_INTERNAL, STATUS_TIMEOUT = 1, 2, 4, 8, 16
_ERR = {SBC_EINVAL: "SBC_EINVAL", SBC_ECAPACITY: "SBC_ECAPACITY", SBC_ENONFINITE: "SBC_ENONFINITE",
        SBC_ECORRUPT: "SBC_ECORRUPT", SBC_ETIMEOUT: "SBC_ETIMEOUT", SBC_ECUDA: "SBC_ECUDA"}

EXPORTS = [
    "sbc_kept_count", "sbc_golomb_b", "sbc_mean_position_bits", "sbc_stream_bytes",
    "sbc_workspace_bytes", "sbc_encode", "sbc_encode_ex", "sbc_encode_launches", "sbc_decode_launches",
    "sbc_encode_diag_get", "sbc_encode_host", "sbc_stream_info_get", "sbc_decode_accumulate",
    "sbc_decode_accumulate_host", "sbc_encode_static", "sbc_workspace_bytes_batch", "sbc_encode_batch",
    "sbc_decode_workspace_bytes_batch", "sbc_decode_accumulate_batch", "sbc_decode_apply", "sbc_stream_bytes_values", "sbc_encode_values", "sbc_stream_bytes_sampled",
    "sbc_workspace_bytes_sampled", "sbc_encode_sampled", "sbc_decode_accumulate_sized", "sbc_decode_apply_sized",
    "sbc_debug_barrier_timeout",
    "sbc_fp4_row_bytes", "sbc_fp4_scale_bytes", "sbc_fp4_workspace_bytes", "sbc_fp4_quantise", "sbc_fp4_dequantise",
    "sbc_fp4_product", "sbc_top_logits", "sbc_distill_loss", "sbc_distill_grad", "sbc_distill_loss_grad",
]
SIDE_VALUES = 2
STATIC_WORKSPACE_BYTES = 8 << 20
MARK_BEGIN, MARK_BOUNDS, MARK_COLLECT, MARK_EXACT, MARK_SELECT, MARK_END, MARK_COUNT = range(7)
MARK_NAMES = ["bounds", "collect", "exact", "select", "golomb"]  # interval i = mark i -> mark i+1


class SbcError(RuntimeError):
    def __init__(self, code: int, where: str):
        super().__init__(f"{where} failed: {_ERR.get(code, code)}")
        self.code = code


class StreamInfo(C.Structure):
    _fields_ = [
        ("magic", C.c_uint32), ("version", C.c_uint32),
        ("numel", C.c_uint64), ("k", C.c_uint64), ("nbits", C.c_uint64), ("payload_offset", C.c_uint64),
        ("b", C.c_uint32), ("side", C.c_uint32), ("mu", C.c_float),
        ("chunk_codewords", C.c_uint32), ("n_chunks", C.c_uint32), ("status", C.c_uint32),
        ("total_bytes", C.c_uint64),
    ]


class EncodeDiag(C.Structure):
    _fields_ = [
        ("status", C.c_uint32), ("exact_route", C.c_uint32), ("candidates", C.c_uint32 * 2),
        ("capacity", C.c_uint32), ("bound_lo", C.c_float), ("bound_hi", C.c_float),
        ("mu_pos", C.c_double), ("mu_neg", C.c_double), ("certain", C.c_uint32 * 2), ("regathered", C.c_uint32),
    ]


class TensorDesc(C.Structure):
    _fields_ = [("update", C.c_void_p), ("residual", C.c_void_p), ("numel", C.c_int64), ("p", C.c_double),
                ("out_stream", C.c_void_p), ("out_capacity", C.c_size_t), ("out_mu", C.c_void_p)]


class Fp4Desc(C.Structure):
    _fields_ = [("values", C.c_void_p), ("scales", C.c_void_p), ("tensor_scale", C.c_void_p), ("rows", C.c_int64),
                ("cols", C.c_int64), ("format", C.c_int32), ("reserved", C.c_int32)]


class DistillDesc(C.Structure):
    _fields_ = [("values", C.c_void_p), ("indices", C.c_void_p), ("rest", C.c_void_p), ("labels", C.c_void_p),
                ("k", C.c_int32), ("temperature", C.c_float), ("alpha", C.c_float), ("reserved", C.c_int32)]


class DecodeDesc(C.Structure):
    _fields_ = [("streams", C.POINTER(C.c_void_p)), ("out_dense", C.c_void_p), ("numel", C.c_int64),
                ("stream_bytes", C.POINTER(C.c_size_t))]


_lib = None


def lib() -> C.CDLL:
    """The loaded CUDA library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_1805_08768_b200.build` "
                "(there is no CPU fallback)")
        L = C.CDLL(LIB_PATH)
        L.sbc_kept_count.restype = C.c_int64
        L.sbc_kept_count.argtypes = [C.c_int64, C.c_double]
        L.sbc_golomb_b.restype = C.c_int
        L.sbc_golomb_b.argtypes = [C.c_double]
        L.sbc_mean_position_bits.restype = C.c_double
        L.sbc_mean_position_bits.argtypes = [C.c_double, C.c_int]
        L.sbc_stream_bytes.restype = C.c_size_t
        L.sbc_stream_bytes.argtypes = [C.c_int64, C.c_double]
        L.sbc_workspace_bytes.restype = C.c_size_t
        L.sbc_workspace_bytes.argtypes = [C.c_int64, C.c_double]
        L.sbc_encode.restype = C.c_int
        L.sbc_encode.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_double, C.c_void_p, C.c_size_t,
                                 C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.sbc_encode_ex.restype = C.c_int
        L.sbc_encode_ex.argtypes = L.sbc_encode.argtypes + [C.POINTER(C.c_void_p)]
        L.sbc_encode_launches.restype = C.c_int
        L.sbc_encode_launches.argtypes = []
        L.sbc_decode_launches.restype = C.c_int
        L.sbc_decode_launches.argtypes = [C.c_int]
        L.sbc_encode_diag_get.restype = C.c_int
        L.sbc_encode_diag_get.argtypes = [C.c_void_p, C.POINTER(EncodeDiag), C.c_void_p]
        L.sbc_encode_host.restype = C.c_int
        L.sbc_encode_host.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_double, C.c_void_p,
                                      C.c_void_p, C.c_size_t, C.POINTER(C.c_size_t), C.POINTER(C.c_float),
                                      C.c_void_p, C.c_size_t, C.c_void_p]
        L.sbc_decode_accumulate_host.restype = C.c_int
        L.sbc_decode_accumulate_host.argtypes = [C.POINTER(C.c_void_p), C.POINTER(C.c_size_t), C.c_int,
                                                 C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_size_t,
                                                 C.POINTER(C.c_uint32), C.c_void_p]
        L.sbc_encode_static.restype = C.c_int
        L.sbc_encode_static.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_double, C.c_void_p, C.c_size_t,
                                        C.c_void_p, C.c_void_p]
        L.sbc_workspace_bytes_batch.restype = C.c_size_t
        L.sbc_workspace_bytes_batch.argtypes = [C.c_int, C.POINTER(TensorDesc)]
        L.sbc_encode_batch.restype = C.c_int
        L.sbc_encode_batch.argtypes = [C.c_int, C.POINTER(TensorDesc), C.c_void_p, C.c_size_t, C.c_void_p]
        L.sbc_decode_workspace_bytes_batch.restype = C.c_size_t
        L.sbc_decode_workspace_bytes_batch.argtypes = [C.c_int]
        L.sbc_decode_accumulate_batch.restype = C.c_int
        L.sbc_decode_accumulate_batch.argtypes = [C.c_int, C.c_int, C.POINTER(DecodeDesc), C.c_void_p, C.c_void_p,
                                                  C.c_size_t, C.c_void_p]
        L.sbc_decode_apply.restype = C.c_int
        L.sbc_decode_apply.argtypes = [C.POINTER(C.c_void_p), C.c_int, C.c_float, C.c_void_p, C.c_void_p, C.c_int64,
                                       C.c_void_p, C.c_void_p]
        L.sbc_stream_bytes_values.restype = C.c_size_t
        L.sbc_stream_bytes_values.argtypes = [C.c_int64, C.c_double]
        L.sbc_encode_values.restype = C.c_int
        L.sbc_encode_values.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_double, C.c_void_p, C.c_size_t,
                                        C.c_void_p, C.c_size_t, C.c_void_p]
        L.sbc_stream_bytes_sampled.restype = C.c_size_t
        L.sbc_stream_bytes_sampled.argtypes = [C.c_int64, C.c_double]
        L.sbc_workspace_bytes_sampled.restype = C.c_size_t
        L.sbc_workspace_bytes_sampled.argtypes = [C.c_int64, C.c_double, C.c_int64]
        L.sbc_encode_sampled.restype = C.c_int
        L.sbc_encode_sampled.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_double, C.c_void_p, C.c_int64,
                                         C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.sbc_stream_info_get.restype = C.c_int
        L.sbc_stream_info_get.argtypes = [C.c_void_p, C.POINTER(StreamInfo), C.c_void_p]
        L.sbc_decode_accumulate.restype = C.c_int
        L.sbc_decode_accumulate.argtypes = [C.POINTER(C.c_void_p), C.c_int, C.c_void_p, C.c_int64,
                                            C.c_void_p, C.c_void_p]
        L.sbc_decode_accumulate_sized.restype = C.c_int
        L.sbc_decode_accumulate_sized.argtypes = [C.POINTER(C.c_void_p), C.POINTER(C.c_size_t), C.c_int, C.c_void_p,
                                                  C.c_int64, C.c_void_p, C.c_void_p]
        L.sbc_decode_apply_sized.restype = C.c_int
        L.sbc_decode_apply_sized.argtypes = [C.POINTER(C.c_void_p), C.POINTER(C.c_size_t), C.c_int, C.c_float,
                                             C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]
        L.sbc_fp4_row_bytes.restype = C.c_size_t
        L.sbc_fp4_row_bytes.argtypes = [C.c_int64]
        L.sbc_fp4_scale_bytes.restype = C.c_size_t
        L.sbc_fp4_scale_bytes.argtypes = [C.c_int64, C.c_int64, C.c_int]
        L.sbc_fp4_workspace_bytes.restype = C.c_size_t
        L.sbc_fp4_workspace_bytes.argtypes = [C.c_int64, C.c_int64, C.c_int]
        L.sbc_fp4_quantise.restype = C.c_int
        L.sbc_fp4_quantise.argtypes = [C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_int64, C.POINTER(Fp4Desc),
                                       C.POINTER(Fp4Desc), C.c_void_p, C.c_size_t, C.c_void_p]
        L.sbc_fp4_dequantise.restype = C.c_int
        L.sbc_fp4_dequantise.argtypes = [C.POINTER(Fp4Desc), C.c_void_p, C.c_int, C.c_int64, C.c_void_p]
        L.sbc_fp4_product.restype = C.c_int
        L.sbc_fp4_product.argtypes = [C.POINTER(Fp4Desc), C.POINTER(Fp4Desc), C.c_void_p, C.c_int, C.c_int64,
                                      C.c_void_p, C.c_void_p]
        L.sbc_top_logits.restype = C.c_int
        L.sbc_top_logits.argtypes = [C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_int64, C.c_int, C.c_float,
                                     C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.sbc_distill_loss.restype = C.c_int
        L.sbc_distill_loss.argtypes = [C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_int64, C.POINTER(DistillDesc),
                                       C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.sbc_distill_grad.restype = C.c_int
        L.sbc_distill_grad.argtypes = [C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_int64, C.POINTER(DistillDesc),
                                       C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p]
        L.sbc_distill_loss_grad.restype = C.c_int
        L.sbc_distill_loss_grad.argtypes = [C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_int64,
                                            C.POINTER(DistillDesc), C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64,
                                            C.c_void_p, C.c_void_p]
        _lib = L
    return _lib


def _check(code: int, where: str) -> None:
    if code != SBC_OK:
        raise SbcError(code, where)


_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _current_stream() -> int:
    return torch.cuda.current_stream().cuda_stream


if hasattr(torch._C, "_cuda_getCurrentRawStream"):   # the same handle without the Stream object around it
    def _current_stream() -> int:  # noqa: F811
        return torch._C._cuda_getCurrentRawStream(_current_device())


def _cuda_stream(stream) -> int:
    if stream is None:
        return _current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _dev_f32(t: torch.Tensor, name: str) -> None:
    if not (t.is_cuda and t.dtype == torch.float32 and t.is_contiguous()):
        raise TypeError(f"{name} must be a contiguous float32 CUDA tensor")


# ---- host-side pure functions --------------------------------------------------

def sbc_kept_count(numel: int, p: float) -> int:
    return int(lib().sbc_kept_count(numel, p))


def sbc_golomb_b(p: float) -> int:
    return int(lib().sbc_golomb_b(p))


def sbc_mean_position_bits(p: float, b: int) -> float:
    return float(lib().sbc_mean_position_bits(p, b))


def sbc_stream_bytes(numel: int, p: float) -> int:
    return int(lib().sbc_stream_bytes(numel, p))


def sbc_workspace_bytes(numel: int, p: float) -> int:
    return int(lib().sbc_workspace_bytes(numel, p))


# ---- device entry points ---------------------------------------------------------

def sbc_encode(update: torch.Tensor, residual: torch.Tensor, p: float,
               out_stream: Optional[torch.Tensor] = None, out_mu: Optional[torch.Tensor] = None,
               workspace: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Enqueue one client step; ``residual`` is updated in place.

    Returns (out_stream uint8 tensor of capacity bytes, out_mu float32[1]),
    both on the device and valid once the CUDA stream has run the work."""
    _dev_f32(update, "update")
    _dev_f32(residual, "residual")
    n = update.numel()
    if residual.numel() != n:
        raise ValueError("update and residual differ in size")
    dev = update.device
    if out_stream is None:
        out_stream = torch.empty(sbc_stream_bytes(n, p), dtype=torch.uint8, device=dev)
    if out_mu is None:
        out_mu = torch.empty(1, dtype=torch.float32, device=dev)
    if workspace is None:
        workspace = torch.empty(sbc_workspace_bytes(n, p), dtype=torch.uint8, device=dev)
    code = lib().sbc_encode(update.data_ptr(), residual.data_ptr(), n, float(p),
                            out_stream.data_ptr(), out_stream.numel(), out_mu.data_ptr(),
                            workspace.data_ptr(), workspace.numel(), _cuda_stream(stream))
    _check(code, "sbc_encode")
    return out_stream, out_mu


def _tensor_descs(updates, residuals, ps, out_streams, out_mus):
    """One sbc_tensor_desc per tensor of a batch (the only place they are marshalled)."""
    n = len(updates)
    descs = (TensorDesc * n)()
    for t in range(n):
        _dev_f32(updates[t], "update")
        _dev_f32(residuals[t], "residual")
        d = descs[t]
        d.update, d.residual, d.numel, d.p = updates[t].data_ptr(), residuals[t].data_ptr(), updates[t].numel(), float(ps[t])
        d.out_stream, d.out_capacity, d.out_mu = out_streams[t].data_ptr(), out_streams[t].numel(), out_mus[t].data_ptr()
    return descs


def _decode_descs(streams_per_tensor, out_denses, sizes_per_tensor=None):
    """One sbc_decode_desc per tensor; returns (descs, n_clients, objects the descs point into)."""
    n = len(out_denses)
    n_clients = len(streams_per_tensor[0])
    descs = (DecodeDesc * n)()
    keep = []
    for t in range(n):
        if len(streams_per_tensor[t]) != n_clients:
            raise ValueError("every tensor needs the same number of client streams")
        _dev_f32(out_denses[t], "out_dense")
        ptrs = (C.c_void_p * n_clients)(*[s.data_ptr() for s in streams_per_tensor[t]])
        keep.append(ptrs)
        descs[t].streams = ptrs
        descs[t].out_dense = out_denses[t].data_ptr()
        descs[t].numel = out_denses[t].numel()
        if sizes_per_tensor is not None:
            lens = (C.c_size_t * n_clients)(*[int(x) for x in sizes_per_tensor[t]])
            keep.append(lens)
            descs[t].stream_bytes = lens
    return descs, n_clients, keep


def sbc_workspace_bytes_batch(numels: Sequence[int], ps: Sequence[float]) -> int:
    n = len(numels)
    descs = (TensorDesc * n)()
    for t in range(n):
        descs[t].numel = int(numels[t])
        descs[t].p = float(ps[t])
    return int(lib().sbc_workspace_bytes_batch(n, descs))


class EncodeBatch:
    """The marshalled descriptors of a batch, built once and reused every round (same tensors)."""

    def __init__(self, updates, residuals, ps, out_streams, out_mus, workspace):
        self.n = len(updates)
        self.descs = _tensor_descs(updates, residuals, ps, out_streams, out_mus)
        self.keep = (list(updates), list(residuals), list(out_streams), list(out_mus), workspace)
        self.ws_ptr, self.ws_bytes = workspace.data_ptr(), workspace.numel()

    def run(self, stream=None) -> None:
        _check(lib().sbc_encode_batch(self.n, self.descs, self.ws_ptr, self.ws_bytes, _cuda_stream(stream)),
               "sbc_encode_batch")


def sbc_encode_batch(updates: Sequence[torch.Tensor], residuals: Sequence[torch.Tensor], ps: Sequence[float],
                     out_streams: Sequence[torch.Tensor], out_mus: Sequence[torch.Tensor],
                     workspace: torch.Tensor, stream=None) -> None:
    """sbc_encode of every tensor of a round with one launch sequence for the whole batch."""
    EncodeBatch(updates, residuals, ps, out_streams, out_mus, workspace).run(stream)


class DecodeBatch:
    """The marshalled descriptors of a batched decode, built once and reused.  ``sizes_per_tensor``
    (readable bytes behind every stream) makes the decoder check each header against them."""

    def __init__(self, streams_per_tensor, out_denses, workspace, status=None, sizes_per_tensor=None):
        self.n = len(out_denses)
        self.descs, self.n_clients, keep = _decode_descs(streams_per_tensor, out_denses, sizes_per_tensor)
        self.keep = [streams_per_tensor, out_denses, workspace, status, keep]
        self.status_ptr = status.data_ptr() if status is not None else None
        self.ws_ptr, self.ws_bytes = workspace.data_ptr(), workspace.numel()

    def run(self, stream=None) -> None:
        _check(lib().sbc_decode_accumulate_batch(self.n, self.n_clients, self.descs, self.status_ptr,
                                                 self.ws_ptr, self.ws_bytes, _cuda_stream(stream)),
               "sbc_decode_accumulate_batch")


def sbc_decode_workspace_bytes_batch(n_tensors: int) -> int:
    return int(lib().sbc_decode_workspace_bytes_batch(n_tensors))


def sbc_decode_accumulate_batch(streams_per_tensor: Sequence[Sequence[torch.Tensor]],
                                out_denses: Sequence[torch.Tensor], workspace: torch.Tensor,
                                status: Optional[torch.Tensor] = None, stream=None, sizes_per_tensor=None) -> None:
    """out_denses[t][j] += mu for every client stream of every tensor t; one launch for the batch."""
    DecodeBatch(streams_per_tensor, out_denses, workspace, status, sizes_per_tensor).run(stream)


def sbc_encode_static(update: torch.Tensor, residual: torch.Tensor, p: float, out_stream: torch.Tensor,
                      out_mu: torch.Tensor, stream=None) -> None:
    """sbc_encode for callers that may not allocate: the scratch is a fixed array inside the
    library (one per GPU, shared by all calls -- do not overlap calls).  The caller passes every
    input and output; problems whose scratch exceeds STATIC_WORKSPACE_BYTES raise SBC_ECAPACITY."""
    _dev_f32(update, "update")
    _dev_f32(residual, "residual")
    code = lib().sbc_encode_static(update.data_ptr(), residual.data_ptr(), update.numel(), float(p),
                                   out_stream.data_ptr(), out_stream.numel(), out_mu.data_ptr(),
                                   _cuda_stream(stream))
    _check(code, "sbc_encode_static")


def sbc_encode_ex(update: torch.Tensor, residual: torch.Tensor, p: float, out_stream: torch.Tensor,
                  out_mu: torch.Tensor, workspace: torch.Tensor, marks: Sequence[torch.cuda.Event],
                  stream=None) -> None:
    """sbc_encode that also records the caller's CUDA events at the stage boundaries."""
    _dev_f32(update, "update")
    _dev_f32(residual, "residual")
    if len(marks) != MARK_COUNT:
        raise ValueError(f"need {MARK_COUNT} events")
    handles = (C.c_void_p * MARK_COUNT)(*[m.cuda_event for m in marks])
    code = lib().sbc_encode_ex(update.data_ptr(), residual.data_ptr(), update.numel(), float(p),
                               out_stream.data_ptr(), out_stream.numel(), out_mu.data_ptr(),
                               workspace.data_ptr(), workspace.numel(), _cuda_stream(stream), handles)
    _check(code, "sbc_encode_ex")


def sbc_encode_launches() -> int:
    return int(lib().sbc_encode_launches())


def sbc_decode_launches(n_clients: int) -> int:
    return int(lib().sbc_decode_launches(n_clients))


def sbc_debug_barrier_timeout(scratch: torch.Tensor, stream=None) -> None:
    """Enqueue the kernel whose barrier cannot be passed; scratch[1] then holds STATUS_TIMEOUT."""
    if not (scratch.is_cuda and scratch.dtype == torch.int32 and scratch.numel() >= 2):
        raise TypeError("scratch must be an int32 CUDA tensor of at least two elements")
    L = lib()
    L.sbc_debug_barrier_timeout.restype = C.c_int
    L.sbc_debug_barrier_timeout.argtypes = [C.c_void_p, C.c_void_p]
    _check(L.sbc_debug_barrier_timeout(scratch.data_ptr(), _cuda_stream(stream)), "sbc_debug_barrier_timeout")


def sbc_encode_diag_get(workspace: torch.Tensor, stream=None) -> EncodeDiag:
    d = EncodeDiag()
    _check(lib().sbc_encode_diag_get(workspace.data_ptr(), C.byref(d), _cuda_stream(stream)),
           "sbc_encode_diag_get")
    return d


def sbc_encode_host(update_host: torch.Tensor, update_dev: torch.Tensor, residual_dev: torch.Tensor,
                    p: float, out_stream_host: torch.Tensor, stream_dev: torch.Tensor,
                    workspace: torch.Tensor, stream=None) -> Tuple[int, float]:
    """Host-buffer encode; synchronises.  Returns (container bytes written, mu)."""
    nbytes, mu = C.c_size_t(), C.c_float()
    code = lib().sbc_encode_host(update_host.data_ptr(), update_dev.data_ptr(), residual_dev.data_ptr(),
                                 update_host.numel(), float(p), out_stream_host.data_ptr(),
                                 stream_dev.data_ptr(), min(stream_dev.numel(), out_stream_host.numel()),
                                 C.byref(nbytes), C.byref(mu), workspace.data_ptr(), workspace.numel(),
                                 _cuda_stream(stream))
    _check(code, "sbc_encode_host")
    return int(nbytes.value), float(mu.value)


def sbc_decode_accumulate_host(streams_host: Sequence[torch.Tensor], sizes: Sequence[int],
                               out_dense_host: torch.Tensor, dense_dev: torch.Tensor,
                               staging_dev: torch.Tensor, stream=None) -> int:
    """Host-buffer decode-and-sum into a zeroed tensor; synchronises.  Returns the status word."""
    nc = len(streams_host)
    ptrs = (C.c_void_p * max(nc, 1))(*[s.data_ptr() for s in streams_host])
    lens = (C.c_size_t * max(nc, 1))(*[int(x) for x in sizes])
    status = C.c_uint32()
    code = lib().sbc_decode_accumulate_host(ptrs, lens, nc, out_dense_host.data_ptr(), dense_dev.data_ptr(),
                                            dense_dev.numel(), staging_dev.data_ptr(), staging_dev.numel(),
                                            C.byref(status), _cuda_stream(stream))
    _check(code, "sbc_decode_accumulate_host")
    return int(status.value)


def sbc_stream_info_get(out_stream: torch.Tensor, stream=None, check: bool = True) -> StreamInfo:
    """Synchronise and read the container header.  With ``check`` a bad status raises."""
    info = StreamInfo()
    code = lib().sbc_stream_info_get(out_stream.data_ptr(), C.byref(info), _cuda_stream(stream))
    if check:
        _check(code, "sbc_stream_info_get")
    return info


def sbc_decode_accumulate(streams: Sequence[torch.Tensor], out_dense: torch.Tensor,
                          status: Optional[torch.Tensor] = None, stream=None,
                          sizes: Optional[Sequence[int]] = None) -> None:
    """Enqueue out_dense[j] += mu_c for every position j of every client stream c.  With ``sizes``
    (readable bytes behind every stream) the _sized entry point checks each header against them."""
    sbc_decode_apply(streams, 1.0, out_dense, None, status, stream, sizes, _plain=True)


def sbc_decode_apply(streams: Sequence[torch.Tensor], scale: float, weights: torch.Tensor,
                     momentum: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                     stream=None, sizes: Optional[Sequence[int]] = None, _plain: bool = False) -> None:
    """Enqueue weights[j] += scale * mu_c at every decoded position; momentum[j] = 0 there."""
    _dev_f32(weights, "weights")
    if momentum is not None:
        _dev_f32(momentum, "momentum")
    nc = len(streams)
    ptrs = (C.c_void_p * max(nc, 1))(*[s.data_ptr() for s in streams])
    st = status.data_ptr() if status is not None else None
    L = lib()
    if sizes is not None:
        if len(sizes) != nc:
            raise ValueError("one size per stream")
        lens = (C.c_size_t * max(nc, 1))(*[int(x) for x in sizes])
        if _plain:
            code = L.sbc_decode_accumulate_sized(ptrs, lens, nc, weights.data_ptr(), weights.numel(), st,
                                                 _cuda_stream(stream))
        else:
            code = L.sbc_decode_apply_sized(ptrs, lens, nc, float(scale), weights.data_ptr(),
                                            momentum.data_ptr() if momentum is not None else None,
                                            weights.numel(), st, _cuda_stream(stream))
    elif _plain:
        code = L.sbc_decode_accumulate(ptrs, nc, weights.data_ptr(), weights.numel(), st, _cuda_stream(stream))
    else:
        code = L.sbc_decode_apply(ptrs, nc, float(scale), weights.data_ptr(),
                                  momentum.data_ptr() if momentum is not None else None, weights.numel(), st,
                                  _cuda_stream(stream))
    _check(code, "sbc_decode_accumulate" if _plain else "sbc_decode_apply")


def sbc_stream_bytes_values(numel: int, p: float) -> int:
    return int(lib().sbc_stream_bytes_values(numel, p))


def sbc_encode_values(update: torch.Tensor, residual: torch.Tensor, p: float,
                      out_stream: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                      stream=None) -> torch.Tensor:
    """Gradient Dropping client step (top-p by magnitude, values sent); residual updated in place."""
    _dev_f32(update, "update")
    _dev_f32(residual, "residual")
    n = update.numel()
    if out_stream is None:
        out_stream = torch.empty(sbc_stream_bytes_values(n, p), dtype=torch.uint8, device=update.device)
    if workspace is None:
        workspace = torch.empty(sbc_workspace_bytes(n, p), dtype=torch.uint8, device=update.device)
    code = lib().sbc_encode_values(update.data_ptr(), residual.data_ptr(), n, float(p), out_stream.data_ptr(),
                                   out_stream.numel(), workspace.data_ptr(), workspace.numel(),
                                   _cuda_stream(stream))
    _check(code, "sbc_encode_values")
    return out_stream


def sbc_stream_bytes_sampled(numel: int, p: float) -> int:
    return int(lib().sbc_stream_bytes_sampled(numel, p))


def sbc_workspace_bytes_sampled(numel: int, p: float, sample_count: int) -> int:
    return int(lib().sbc_workspace_bytes_sampled(numel, p, sample_count))


def sbc_encode_sampled(update: torch.Tensor, residual: torch.Tensor, p: float, sample_idx: torch.Tensor,
                       out_stream: Optional[torch.Tensor] = None, out_mu: Optional[torch.Tensor] = None,
                       workspace: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """sbc_encode with the two thresholds taken from the caller's subsample (int32 CUDA positions)."""
    _dev_f32(update, "update")
    _dev_f32(residual, "residual")
    if not (sample_idx.is_cuda and sample_idx.dtype == torch.int32 and sample_idx.is_contiguous()):
        raise TypeError("sample_idx must be a contiguous int32 CUDA tensor")
    n, m = update.numel(), sample_idx.numel()
    dev = update.device
    if out_stream is None:
        out_stream = torch.empty(sbc_stream_bytes_sampled(n, p), dtype=torch.uint8, device=dev)
    if out_mu is None:
        out_mu = torch.empty(1, dtype=torch.float32, device=dev)
    if workspace is None:
        workspace = torch.empty(sbc_workspace_bytes_sampled(n, p, m), dtype=torch.uint8, device=dev)
    code = lib().sbc_encode_sampled(update.data_ptr(), residual.data_ptr(), n, float(p), sample_idx.data_ptr(), m,
                                    out_stream.data_ptr(), out_stream.numel(), out_mu.data_ptr(),
                                    workspace.data_ptr(), workspace.numel(), _cuda_stream(stream))
    _check(code, "sbc_encode_sampled")
    return out_stream, out_mu


# ---- language-model operators (include/sbc_lm.h) -----------------------------------

DTYPE_CODES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
FP4_WORKSPACE_BYTES = 4096   # what sbc_fp4_workspace_bytes says for any matrix
FP4_FORMATS = {"e8m0": 0, "e4m3": 1}   # block scales: powers of two for 32 elements, 8-bit floats for 16


def _matrix(t: torch.Tensor, name: str) -> Tuple[int, int, int, int]:
    """(rows, columns, elements between rows, type code) of a matrix argument."""
    code = DTYPE_CODES.get(t.dtype)
    if code is None or not t.is_cuda or t.dim() != 2:
        raise TypeError(f"{name} must be a float32, bfloat16 or float16 CUDA matrix")
    if t.get_device() != _current_device():
        raise ValueError(f"{name} is on {t.device}, the current device is cuda:{_current_device()}")
    rows, cols = t.shape
    across, along = t.stride()
    if cols > 1 and along != 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    if rows <= 1:
        across = max(cols, 1)
    elif across < cols:
        raise ValueError(f"{name}: rows must not overlap")
    return rows, cols, across, code


def _beside(t: torch.Tensor, other: torch.Tensor, name: str) -> None:
    if t.get_device() != other.get_device():
        raise ValueError(f"{name} is on {t.device}, not on {other.device}")


def _status(status: Optional[torch.Tensor], other: torch.Tensor) -> Optional[int]:
    if status is None:
        return None
    if not (status.is_cuda and status.dtype == torch.int32 and status.numel() >= 1):
        raise TypeError("status must be an int32 CUDA tensor")
    _beside(status, other, "status")
    return status.data_ptr()


def _empty(stream, shape, dtype, like: torch.Tensor) -> torch.Tensor:
    """A new buffer beside `like` that belongs to the stream which the work is enqueued on."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    s = stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(_cuda_stream(stream))
    with torch.cuda.stream(s):
        return like.new_empty(shape, dtype=dtype)


def _fp4_sizes(rows: int, cols: int, format: str) -> Tuple[int, int]:
    """(bytes of the elements, bytes of the scales), as the header lays them out."""
    if format not in FP4_FORMATS:
        raise ValueError(f"unknown 4-bit format {format!r}")
    if rows < 1 or cols < 1:
        raise ValueError("an Fp4Tensor has at least one row and one column")
    tiles = (cols + 127) // 128 if format == "e8m0" else (cols + 63) // 64
    return rows * ((cols + 31) // 32 * 16), (rows + 127) // 128 * tiles * 512


class Fp4Tensor:
    """A matrix (rows x cols) in 4-bit floating point with a scale per block; the layout is the C
    header's.  ``values`` uint8 [rows, row bytes], ``scales`` uint8 (flat), ``tensor_scale`` float32 [1];
    ``format`` is "e8m0" or "e4m3"."""

    __slots__ = ("rows", "cols", "format", "desc", "_room", "_at", "_parts", "_device")

    def __init__(self, values: torch.Tensor, scales: torch.Tensor, tensor_scale: torch.Tensor, rows: int, cols: int,
                 format: str):
        value_bytes, scale_bytes = _fp4_sizes(rows, cols, format)
        for t, name, n in ((values, "values", value_bytes), (scales, "scales", scale_bytes)):
            if not (t.is_cuda and t.dtype == torch.uint8 and t.is_contiguous()):
                raise TypeError(f"{name} must be a contiguous uint8 CUDA tensor")
            if t.numel() != n:
                raise ValueError(f"{name}: {n} bytes needed for {rows} x {cols}, got {t.numel()}")
        _dev_f32(tensor_scale, "tensor_scale")
        _beside(scales, values, "scales")
        _beside(tensor_scale, values, "tensor_scale")
        if tensor_scale.numel() < 1:
            raise ValueError("tensor_scale must hold one value")
        self.rows, self.cols, self.format = rows, cols, format
        self._room, self._at, self._parts = None, 0, (values, scales, tensor_scale)
        self._device = values.get_device()
        self.desc = Fp4Desc(values.data_ptr(), scales.data_ptr(), tensor_scale.data_ptr(), rows, cols,
                            FP4_FORMATS[format], 0)

    @classmethod
    def _in_room(cls, room: torch.Tensor, at: int, value_bytes: int, scale_bytes: int, rows: int, cols: int,
                 format: str) -> "Fp4Tensor":
        """Elements, scales and tensor scale one behind the other in a byte buffer."""
        self = cls.__new__(cls)
        self.rows, self.cols, self.format = rows, cols, format
        self._room, self._at, self._parts = room, at, None
        self._device = room.get_device()
        base = room.data_ptr() + at
        self.desc = Fp4Desc(base, base + value_bytes, base + value_bytes + scale_bytes, rows, cols,
                            FP4_FORMATS[format], 0)
        return self

    @classmethod
    def empty(cls, rows: int, cols: int, format: str, device, stream=None) -> "Fp4Tensor":
        """Room for a rows x cols matrix, contents undefined."""
        value_bytes, scale_bytes = _fp4_sizes(rows, cols, format)
        if stream is not None:
            with torch.cuda.stream(stream):
                return cls.empty(rows, cols, format, device)
        room = torch.empty(value_bytes + scale_bytes + 16, dtype=torch.uint8, device=device)
        return cls._in_room(room, 0, value_bytes, scale_bytes, rows, cols, format)

    def _views(self):
        if self._parts is None:
            value_bytes, scale_bytes = _fp4_sizes(self.rows, self.cols, self.format)
            a, b = self._at, self._at + value_bytes
            self._parts = (self._room[a:b].view(self.rows, -1), self._room[b:b + scale_bytes],
                           self._room[b + scale_bytes:b + scale_bytes + 4].view(torch.float32))
        return self._parts

    values = property(lambda self: self._views()[0])
    scales = property(lambda self: self._views()[1])
    tensor_scale = property(lambda self: self._views()[2])

    @property
    def _any(self) -> torch.Tensor:
        return self._room if self._room is not None else self._parts[0]

    @property
    def device(self) -> torch.device:
        return self._any.device

    @property
    def nbytes(self) -> int:
        return sum(_fp4_sizes(self.rows, self.cols, self.format)) + 4


def _quantise(x, format, along_rows, along_cols, stream):
    rows, cols, across, code = _matrix(x, "x")
    # one buffer: both tensors and, in front, the scratch of the call
    at_t = ws = FP4_WORKSPACE_BYTES
    v = s = v_t = s_t = 0
    if along_rows:
        v, s = _fp4_sizes(rows, cols, format)
        at_t += v + s + 16
    if along_cols:
        v_t, s_t = _fp4_sizes(cols, rows, format)
    room = _empty(stream, at_t + (v_t + s_t + 16 if along_cols else 0), torch.uint8, x)
    q = Fp4Tensor._in_room(room, ws, v, s, rows, cols, format) if along_rows else None
    q_t = Fp4Tensor._in_room(room, at_t, v_t, s_t, cols, rows, format) if along_cols else None
    rc = lib().sbc_fp4_quantise(x.data_ptr(), code, rows, cols, across, C.byref(q.desc) if along_rows else None,
                                C.byref(q_t.desc) if along_cols else None, room.data_ptr(), ws, _cuda_stream(stream))
    if rc:
        _check(rc, "sbc_fp4_quantise")
    return q, q_t


def sbc_fp4_quantise(x: torch.Tensor, format: str = "e8m0", transposed: bool = False, stream=None) -> Fp4Tensor:
    """x (rows x cols) in 4 bits, blocks along its rows; with ``transposed`` its transpose (cols x rows),
    blocks down the columns of x."""
    return _quantise(x, format, not transposed, transposed, stream)[1 if transposed else 0]


def sbc_fp4_quantise_both(x: torch.Tensor, format: str = "e8m0", stream=None) -> Tuple[Fp4Tensor, Fp4Tensor]:
    """(x in 4 bits along its rows, its transpose in 4 bits), x read once: what a forward and a
    backward product contract."""
    return _quantise(x, format, True, True, stream)


def sbc_fp4_dequantise(q: Fp4Tensor, dtype: torch.dtype = torch.float32, out: Optional[torch.Tensor] = None,
                       stream=None) -> torch.Tensor:
    """The values that q stands for (rows x cols)."""
    if out is None:
        out = _empty(stream, (q.rows, q.cols), dtype, q._any)
    rows, cols, across, code = _matrix(out, "out")
    if (rows, cols) != (q.rows, q.cols):
        raise ValueError(f"out must be {q.rows} x {q.cols}")
    if q._device != out.get_device():
        raise ValueError("out must be on the tensor's device")
    rc = lib().sbc_fp4_dequantise(C.byref(q.desc), out.data_ptr(), code, across, _cuda_stream(stream))
    if rc:
        _check(rc, "sbc_fp4_dequantise")
    return out


def sbc_fp4_product(a: Fp4Tensor, b: Fp4Tensor, dtype: torch.dtype = torch.bfloat16,
                    out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                    stream=None) -> torch.Tensor:
    """a b^T (a.rows x b.rows): tokens times weights, both in 4 bits, sums in 32 bits."""
    if a.format != b.format or a.cols != b.cols:
        raise ValueError(f"operands differ: {a.cols} columns of {a.format}, {b.cols} of {b.format}")
    if out is None:
        out = _empty(stream, (a.rows, b.rows), dtype, a._any)
    rows, cols, across, code = _matrix(out, "out")
    if (rows, cols) != (a.rows, b.rows):
        raise ValueError(f"out must be {a.rows} x {b.rows}")
    if not out.get_device() == a._device == b._device:
        raise ValueError("operands and result must be on one device")
    rc = lib().sbc_fp4_product(C.byref(a.desc), C.byref(b.desc), out.data_ptr(), code, across, _status(status, out),
                               _cuda_stream(stream))
    if rc:
        _check(rc, "sbc_fp4_product")
    return out


TOP_MOST, DISTILL_MOST, DISTILL_COLS, DISTILL_STATS = 256, 1024, 1 << 20, 8


def sbc_top_logits(logits: torch.Tensor, k: int, temperature: float = 1.0,
                   stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(values float32 [rows, k], indices int32 [rows, k], rest float32 [rows]): every row's k largest
    logits in descending order and log sum exp(z / temperature) of all the others."""
    rows, cols, across, code = _matrix(logits, "logits")
    if not 1 <= k <= min(cols, TOP_MOST):
        raise ValueError(f"k must be in 1 .. {min(cols, TOP_MOST)}")
    values = _empty(stream, (rows, k), torch.float32, logits)
    indices = _empty(stream, (rows, k), torch.int32, logits)
    rest = _empty(stream, rows, torch.float32, logits)
    rc = lib().sbc_top_logits(logits.data_ptr(), code, rows, cols, across, k, temperature, values.data_ptr(),
                              indices.data_ptr(), rest.data_ptr(), _cuda_stream(stream))
    if rc:
        _check(rc, "sbc_top_logits")
    return values, indices, rest


def _rows_of(t: Optional[torch.Tensor], rows: int, dtype: torch.dtype, name: str, other: torch.Tensor) -> Optional[int]:
    if t is None:
        return None
    if not (t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise TypeError(f"{name} must be a contiguous {dtype} CUDA tensor")
    if t.numel() != rows:
        raise ValueError(f"{name} must hold one value per row")
    _beside(t, other, name)
    return t.data_ptr()


def _taught(logits, values, indices, rest, temperature, alpha, labels):
    """(rows, columns, elements between rows, type code, the teacher's side) of a loss's arguments."""
    rows, cols, across, code = _matrix(logits, "logits")
    _dev_f32(values, "values")
    if not (indices.is_cuda and indices.dtype == torch.int32 and indices.is_contiguous()):
        raise TypeError("indices must be a contiguous int32 CUDA tensor")
    shape = values.shape
    if len(shape) != 2 or shape != indices.shape or shape[0] != rows:
        raise ValueError("values and indices must be rows x k")
    _beside(values, logits, "values")
    _beside(indices, logits, "indices")
    if not 1 <= shape[1] <= DISTILL_MOST:
        raise ValueError(f"k must be in 1 .. {DISTILL_MOST}")
    if not 1 <= cols <= DISTILL_COLS:
        raise ValueError(f"logits must have 1 .. {DISTILL_COLS} columns")
    d = DistillDesc(values.data_ptr(), indices.data_ptr(), _rows_of(rest, rows, torch.float32, "rest", logits),
                    _rows_of(labels, rows, torch.int64, "labels", logits), shape[1], temperature, alpha, 0)
    return rows, cols, across, code, d


def _grad_out(logits: torch.Tensor, out: Optional[torch.Tensor], stream) -> Tuple[torch.Tensor, int]:
    """(the gradient's buffer, elements between its rows)"""
    if out is None:
        return _empty(stream, logits.shape, logits.dtype, logits), max(logits.shape[1], 1)
    across = _matrix(out, "out")[2]
    if out.shape != logits.shape or out.dtype != logits.dtype:
        raise ValueError("out must have the logits' shape and type")
    return out, across


def sbc_distill_loss(logits: torch.Tensor, values: torch.Tensor, indices: torch.Tensor,
                     rest: Optional[torch.Tensor] = None, temperature: float = 1.0, alpha: float = 1.0,
                     labels: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                     stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(loss [rows], statistics for sbc_distill_grad): alpha temperature^2 KL(teacher || student) over the
    sent words and one outcome for all others, plus (1 - alpha) cross entropy of the labels."""
    rows, cols, across, code, d = _taught(logits, values, indices, rest, temperature, alpha, labels)
    loss = _empty(stream, rows, torch.float32, logits)
    stats = _empty(stream, (rows, DISTILL_STATS), torch.float32, logits)
    rc = lib().sbc_distill_loss(logits.data_ptr(), code, rows, cols, across, C.byref(d), loss.data_ptr(),
                                stats.data_ptr(), _status(status, logits), _cuda_stream(stream))
    if rc:
        _check(rc, "sbc_distill_loss")
    return loss, stats


def sbc_distill_grad(logits: torch.Tensor, values: torch.Tensor, indices: torch.Tensor, stats: torch.Tensor,
                     grad_loss: Optional[torch.Tensor] = None, rest: Optional[torch.Tensor] = None,
                     temperature: float = 1.0, alpha: float = 1.0, labels: Optional[torch.Tensor] = None,
                     out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """grad_loss[r] * d loss[r] / d logits[r, :] in the logits' type; ``out`` may be the logits."""
    rows, cols, across, code, d = _taught(logits, values, indices, rest, temperature, alpha, labels)
    out, out_across = _grad_out(logits, out, stream)
    rc = lib().sbc_distill_grad(logits.data_ptr(), code, rows, cols, across, C.byref(d),
                                _rows_of(stats, rows * DISTILL_STATS, torch.float32, "stats", logits),
                                _rows_of(grad_loss, rows, torch.float32, "grad_loss", logits), out.data_ptr(),
                                out_across, _cuda_stream(stream))
    if rc:
        _check(rc, "sbc_distill_grad")
    return out


def sbc_distill_loss_grad(logits: torch.Tensor, values: torch.Tensor, indices: torch.Tensor,
                          grad_loss: Optional[torch.Tensor] = None, rest: Optional[torch.Tensor] = None,
                          temperature: float = 1.0, alpha: float = 1.0, labels: Optional[torch.Tensor] = None,
                          out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                          stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(loss [rows], its gradient times grad_loss) in one reading of the logits; ``out`` may be the logits."""
    rows, cols, across, code, d = _taught(logits, values, indices, rest, temperature, alpha, labels)
    out, out_across = _grad_out(logits, out, stream)
    loss = _empty(stream, rows, torch.float32, logits)
    rc = lib().sbc_distill_loss_grad(logits.data_ptr(), code, rows, cols, across, C.byref(d),
                                     _rows_of(grad_loss, rows, torch.float32, "grad_loss", logits), loss.data_ptr(),
                                     out.data_ptr(), out_across, _status(status, logits), _cuda_stream(stream))
    if rc:
        _check(rc, "sbc_distill_loss_grad")
    return loss, out
