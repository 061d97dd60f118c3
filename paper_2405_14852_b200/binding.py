"""ctypes binding of libpvt.so: argument marshalling only.

Every step of the V step (norms, selection, target formation, search, code
write, dequantisation) runs in the CUDA kernels behind the C ABI declared in
``include/pvt.h``; this module only turns torch tensors into pointers and sizes.
There is no CPU fallback: if the library cannot be loaded, or a call is rejected,
an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional

import torch

from . import build as _build

PVT_F32, PVT_F16, PVT_BF16 = 0, 1, 2
PVT_U8, PVT_U16 = 0, 1
PVT_OK, PVT_EINVAL, PVT_EUNSUPPORTED, PVT_EWORKSPACE, PVT_ECUDA, PVT_ETOOLARGE = 0, -1, -2, -3, -4, -5
PVT_NOALLOC_MAX_GROUPS = 1 << 21
PVT_DEV_BAD_INDEX, PVT_DEV_BAD_CODE, PVT_DEV_WAIT_EXPIRED, PVT_DEV_INTERNAL = 1, 2, 4, 8
PVT_KERNEL_SELECT, PVT_KERNEL_ENCODE_MAIN, PVT_KERNEL_ENCODE_AUX, PVT_KERNEL_DEQUANT = 0, 1, 2, 3
PVT_KERNEL_ENCODE_RESCORE = 4
PVT_KERNEL_PSTEP_GRAD, PVT_KERNEL_ADAM, PVT_KERNEL_TRUST, PVT_KERNEL_REFINE = 5, 6, 7, 8
PVT_KERNEL_MX, PVT_KERNEL_DISTILL, PVT_KERNEL_NORM = 9, 10, 11
PVT_M1_AUTO, PVT_M1_FP32, PVT_M1_TENSOR = 0, 1, 2
PVT_SAMPLE_UNIFORM, PVT_SAMPLE_PROPORTIONAL = 0, 1
PVT_MX_E8M0_32, PVT_MX_E4M3_16 = 0, 1
PVT_DISTILL_MAX_K, PVT_DISTILL_MAX_VOCAB, PVT_DISTILL_STATS = 1024, 1 << 20, 8
PVT_ACT_SILU, PVT_ACT_GELU, PVT_ACT_GELU_TANH = 0, 1, 2
PVT_NORM_LAYER, PVT_NORM_RMS, PVT_NORM_MAX_COLS, PVT_F64 = 0, 1, 32768, 3


_OUT_DTYPE = {torch.float32: PVT_F32, torch.float16: PVT_F16}


class pvt_layer(ctypes.Structure):
    _fields_ = [
        ("rows", ctypes.c_int32), ("cols", ctypes.c_int32), ("group_dim", ctypes.c_int32),
        ("num_codebooks", ctypes.c_int32), ("codebook_size", ctypes.c_int32),
        ("codebook_dtype", ctypes.c_int32), ("code_dtype", ctypes.c_int32), ("beam", ctypes.c_int32),
        ("eta", ctypes.c_float), ("reserved_", ctypes.c_int32),
        ("W", ctypes.c_void_p), ("g", ctypes.c_void_p), ("scale", ctypes.c_void_p),
        ("codebooks", ctypes.c_void_p), ("codes", ctypes.c_void_p),
    ]


class pvt_mx(ctypes.Structure):
    _fields_ = [
        ("rows", ctypes.c_int32), ("cols", ctypes.c_int32), ("format", ctypes.c_int32), ("reserved_", ctypes.c_int32),
        ("ld", ctypes.c_int64), ("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("tensor_scale", ctypes.c_void_p),
    ]


class pvt_distill(ctypes.Structure):
    _fields_ = [
        ("rows", ctypes.c_int64), ("vocab", ctypes.c_int32), ("k", ctypes.c_int32), ("logits", ctypes.c_void_p),
        ("ld", ctypes.c_int64), ("dtype", ctypes.c_int32), ("temperature", ctypes.c_float),
        ("top_idx", ctypes.c_void_p), ("top_logit", ctypes.c_void_p), ("teacher_lse", ctypes.c_void_p),
        ("weight", ctypes.c_void_p),
    ]


class pvt_norm(ctypes.Structure):
    _fields_ = [
        ("rows", ctypes.c_int64), ("cols", ctypes.c_int32), ("kind", ctypes.c_int32), ("x", ctypes.c_void_p),
        ("ldx", ctypes.c_int64), ("residual", ctypes.c_void_p), ("ldr", ctypes.c_int64), ("weight", ctypes.c_void_p),
        ("bias", ctypes.c_void_p), ("dtype", ctypes.c_int32), ("weight_dtype", ctypes.c_int32), ("eps", ctypes.c_float),
        ("reserved_", ctypes.c_int32),
    ]


class PvtError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {strerror(code)} (code {code})" + (f": {last_cuda_error()}" if code == PVT_ECUDA else ""))
        self.code = code


_lib = None


def library_path() -> str:
    return _build.LIB


def lib():
    """The loaded C library.  Builds it in-tree if nvcc is available and the
    shared object is missing or stale; raises if it cannot be loaded."""
    global _lib
    if _lib is None:
        path = library_path()
        if _build.needs_build():
            try:
                _build.build()
            except Exception as exc:  # no compiler on this machine: use the shipped object if there is one
                if not os.path.exists(path):
                    raise RuntimeError(f"libpvt.so is missing and could not be built: {exc}") from exc
        L = ctypes.CDLL(path)
        vp, u64, sz, fl = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_size_t, ctypes.c_float
        lp = ctypes.POINTER(pvt_layer)
        L.pvt_workspace_bytes.restype = sz
        L.pvt_workspace_bytes.argtypes = [lp, u64]
        L.pvt_workspace_init.restype = ctypes.c_int
        L.pvt_workspace_init.argtypes = [vp, sz, vp]
        L.pvt_vstep_select.restype = ctypes.c_int
        L.pvt_vstep_select.argtypes = [lp, u64, vp, vp, sz, vp]
        L.pvt_vstep_select_noalloc.restype = ctypes.c_int
        L.pvt_vstep_select_noalloc.argtypes = [lp, u64, vp, vp, vp]
        L.pvt_vstep_select_ste.restype = ctypes.c_int
        L.pvt_vstep_select_ste.argtypes = [lp, vp, u64, vp, vp, sz, vp]
        L.pvt_vstep_sample.restype = ctypes.c_int
        L.pvt_vstep_sample.argtypes = [lp, u64, ctypes.c_int32, u64, vp, vp, sz, vp]
        L.pvt_vstep_encode.restype = ctypes.c_int
        L.pvt_vstep_encode.argtypes = [lp, vp, u64, vp, vp, sz, vp]
        L.pvt_trust_workspace_bytes.restype = sz
        L.pvt_trust_workspace_bytes.argtypes = [lp, u64]
        L.pvt_vstep_trust.restype = ctypes.c_int
        L.pvt_vstep_trust.argtypes = [lp, u64, fl, vp, vp, vp, vp, sz, vp]
        L.pvt_vstep_refine.restype = ctypes.c_int
        L.pvt_vstep_refine.argtypes = [lp, vp, u64, ctypes.c_int32, vp, vp, vp, vp]
        L.pvt_block_workspace_bytes.restype = sz
        L.pvt_block_workspace_bytes.argtypes = [lp, ctypes.POINTER(u64), ctypes.c_int32]
        L.pvt_vstep_block.restype = ctypes.c_int
        L.pvt_vstep_block.argtypes = [lp, ctypes.POINTER(u64), ctypes.c_int32, ctypes.POINTER(vp), ctypes.POINTER(vp),
                                      ctypes.c_int32, vp, sz, vp]
        L.pvt_dequant.restype = ctypes.c_int
        L.pvt_dequant.argtypes = [lp, vp, ctypes.c_int32, vp, vp]
        i32, i64 = ctypes.c_int32, ctypes.c_int64
        mp = dp = vp  # descriptors: a structure by reference, or its bytes
        L.pvt_mx_scale_bytes.restype = sz
        L.pvt_mx_scale_bytes.argtypes = [i32, i32, i32]
        L.pvt_mx_quantize.restype = ctypes.c_int
        L.pvt_mx_quantize.argtypes = [mp, vp, i32, i64, vp]
        L.pvt_mx_dequant.restype = ctypes.c_int
        L.pvt_mx_dequant.argtypes = [mp, vp, i32, i64, vp]
        L.pvt_mx_product.restype = ctypes.c_int
        L.pvt_mx_product.argtypes = [mp, mp, vp, i32, i64, vp, vp]
        L.pvt_mx_grad_input.restype = ctypes.c_int
        L.pvt_mx_grad_input.argtypes = [vp, i64, i32, mp, vp, i32, i64, vp, vp]
        L.pvt_mx_grad_weight.restype = ctypes.c_int
        L.pvt_mx_grad_weight.argtypes = [vp, i64, i32, mp, vp, i64, i32, vp, vp]
        L.pvt_distill_top.restype = ctypes.c_int
        L.pvt_distill_top.argtypes = [vp, i32, i64, i64, i32, i32, fl, vp, vp, vp, vp]
        L.pvt_distill_loss.restype = ctypes.c_int
        L.pvt_distill_loss.argtypes = [dp, vp, vp, vp, vp, i32, i64, vp, vp]
        L.pvt_distill_grad.restype = ctypes.c_int
        L.pvt_distill_grad.argtypes = [dp, vp, vp, vp, i32, i64, vp, vp]
        L.pvt_mx_gated.restype = ctypes.c_int
        L.pvt_mx_gated.argtypes = [mp, mp, mp, i32, vp, i32, i64, mp, vp, vp]
        L.pvt_mx_gated_grad.restype = ctypes.c_int
        L.pvt_mx_gated_grad.argtypes = [mp, mp, mp, i32, vp, i32, i64, vp, vp, i64, vp, vp]
        L.pvt_mx_gated_grad_input.restype = ctypes.c_int
        L.pvt_mx_gated_grad_input.argtypes = [vp, vp, i64, i32, mp, mp, vp, i32, i64, vp, vp]
        L.pvt_norm_apply.restype = ctypes.c_int
        L.pvt_norm_apply.argtypes = [dp, vp, i64, vp, i32, i64, mp, vp, vp]
        L.pvt_norm_workspace_bytes.restype = sz
        L.pvt_norm_workspace_bytes.argtypes = [dp]
        L.pvt_norm_grad.restype = ctypes.c_int
        L.pvt_norm_grad.argtypes = [dp, vp, i32, vp, i64, vp, i64, vp, i64, vp, vp, i32, i32, vp, sz, vp]
        L.pvt_pstep_grad.restype = ctypes.c_int
        L.pvt_pstep_grad.argtypes = [lp, vp, vp, vp, vp]
        L.pvt_adam_update.restype = ctypes.c_int
        L.pvt_adam_update.argtypes = [vp, vp, vp, vp, vp, u64, fl, fl, fl, fl, fl, fl, vp]
        L.pvt_adam_direction.restype = ctypes.c_int
        L.pvt_adam_direction.argtypes = [vp, vp, vp, vp, u64, fl, fl, fl, fl, fl, vp]
        L.pvt_adam_bias.restype = ctypes.c_int
        L.pvt_adam_bias.argtypes = [u64, fl, fl, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_float)]
        L.pvt_test_wait_limit.restype = None
        L.pvt_test_wait_limit.argtypes = [ctypes.c_uint32, ctypes.c_int64]
        L.pvt_status.restype = ctypes.c_int
        L.pvt_status.argtypes = [vp, vp]
        L.pvt_strerror.restype = ctypes.c_char_p
        L.pvt_strerror.argtypes = [ctypes.c_int]
        L.pvt_last_cuda_error.restype = ctypes.c_char_p
        L.pvt_version.restype = ctypes.c_int
        L.pvt_set_m1_search.restype = None
        L.pvt_set_m1_search.argtypes = [ctypes.c_int]
        L.pvt_timing_enable.restype = None
        L.pvt_timing_enable.argtypes = [ctypes.c_int]
        L.pvt_probe_fp32_tflops.restype = ctypes.c_int
        L.pvt_probe_fp32_tflops.argtypes = [vp, sz, ctypes.POINTER(ctypes.c_float), vp]
        L.pvt_launch_count.restype = ctypes.c_ulonglong
        L.pvt_search_counts.restype = sz
        L.pvt_search_counts.argtypes = [lp, u64]
        L.pvt_timing_read.restype = ctypes.c_int
        L.pvt_timing_read.argtypes = [ctypes.c_int, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_int)]
        _lib = L
    return _lib


def strerror(code: int) -> str:
    return lib().pvt_strerror(code).decode()


def last_cuda_error() -> str:
    return lib().pvt_last_cuda_error().decode()


def _check(code: int, what: str) -> None:
    if code != PVT_OK:
        raise PvtError(code, what)


# the current stream's handle without building a Stream object, where this torch has that query
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_ptr(stream: Optional[torch.cuda.Stream]) -> int:
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def make_layer(rows: int, cols: int, W, g, scale, codebooks, codes, *, eta: float = 1.0, beam: int = 8,
               group_dim: int = 8) -> pvt_layer:
    """Describe a layer whose arrays are CUDA tensors (any of W, g, scale may be
    None for calls that do not read them).  codebooks: [M, K, 8] float32/float16;
    codes: [G, M] uint8/uint16."""
    M, K = int(codebooks.shape[0]), int(codebooks.shape[1])
    for t in (W, g, scale, codebooks, codes):
        if t is not None and (not t.is_cuda or not t.is_contiguous()):
            raise ValueError("layer tensors must be contiguous CUDA tensors")
    cb_dtype = {torch.float32: PVT_F32, torch.float16: PVT_F16}[codebooks.dtype]
    code_dtype = {torch.uint8: PVT_U8, torch.uint16: PVT_U16, torch.int16: PVT_U16}[codes.dtype]
    return pvt_layer(rows, cols, group_dim, M, K, cb_dtype, code_dtype, beam, float(eta), 0,
                     _ptr(W), _ptr(g), _ptr(scale), _ptr(codebooks), _ptr(codes))


def pvt_workspace_bytes(layer: pvt_layer, k: int) -> int:
    n = int(lib().pvt_workspace_bytes(ctypes.byref(layer), k))
    if n == 0:
        raise PvtError(PVT_EINVAL, "pvt_workspace_bytes")
    return n


def pvt_workspace_init(ws: torch.Tensor, stream=None) -> None:
    _check(lib().pvt_workspace_init(ws.data_ptr(), ws.numel() * ws.element_size(), _stream_ptr(stream)),
           "pvt_workspace_init")


def new_workspace(layer: pvt_layer, k: int, device=None) -> torch.Tensor:
    ws = torch.empty(pvt_workspace_bytes(layer, k), dtype=torch.uint8, device=device or "cuda")
    pvt_workspace_init(ws)
    return ws


def pvt_vstep_select(layer: pvt_layer, k: int, idx_out: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
    _check(lib().pvt_vstep_select(ctypes.byref(layer), k, idx_out.data_ptr(), ws.data_ptr(),
                                  ws.numel() * ws.element_size(), _stream_ptr(stream)), "pvt_vstep_select")


def pvt_vstep_select_noalloc(layer: pvt_layer, k: int, idx_out: torch.Tensor,
                             status_out: Optional[torch.Tensor] = None, stream=None) -> None:
    """pvt_vstep_select without a workspace argument: for callers that cannot
    allocate device memory (frozen memory pool, host application owning the
    device memory, allocator-free thread).  The scratch is a fixed array inside
    the library, so the layer may have at most PVT_NOALLOC_MAX_GROUPS groups, and
    calls that could overlap on the GPU must be ordered by the caller."""
    _check(lib().pvt_vstep_select_noalloc(ctypes.byref(layer), k, idx_out.data_ptr(), _ptr(status_out),
                                          _stream_ptr(stream)), "pvt_vstep_select_noalloc")


def pvt_vstep_select_ste(layer: pvt_layer, buffer: torch.Tensor, k: int, idx_out: torch.Tensor, ws: torch.Tensor,
                         stream=None) -> None:
    """pvt_vstep_select that also lets the straight-through buffer (float32 [rows, cols], in place) take the
    step -eta * g (Appendix E)."""
    if buffer.dtype != torch.float32 or not buffer.is_cuda or not buffer.is_contiguous():
        raise ValueError("buffer must be a contiguous float32 CUDA tensor")
    _check(lib().pvt_vstep_select_ste(ctypes.byref(layer), buffer.data_ptr(), k, idx_out.data_ptr(), ws.data_ptr(),
                                      ws.numel() * ws.element_size(), _stream_ptr(stream)), "pvt_vstep_select_ste")


def pvt_vstep_sample(layer: pvt_layer, k: int, rule: int, seed: int, idx_out: torch.Tensor, ws: torch.Tensor,
                     stream=None) -> None:
    """A random subspace of k groups: PVT_SAMPLE_UNIFORM or PVT_SAMPLE_PROPORTIONAL (to the squared update norm)."""
    _check(lib().pvt_vstep_sample(ctypes.byref(layer), k, rule, seed, idx_out.data_ptr(), ws.data_ptr(),
                                  ws.numel() * ws.element_size(), _stream_ptr(stream)), "pvt_vstep_sample")


def pvt_vstep_encode(layer: pvt_layer, idx: torch.Tensor, k: int, err_out: Optional[torch.Tensor],
                     ws: torch.Tensor, stream=None) -> None:
    _check(lib().pvt_vstep_encode(ctypes.byref(layer), idx.data_ptr(), k, _ptr(err_out), ws.data_ptr(),
                                  ws.numel() * ws.element_size(), _stream_ptr(stream)), "pvt_vstep_encode")


def pvt_trust_workspace_bytes(layer: pvt_layer, k_max: int) -> int:
    n = int(lib().pvt_trust_workspace_bytes(ctypes.byref(layer), k_max))
    if n == 0:
        raise PvtError(PVT_EINVAL, "pvt_trust_workspace_bytes")
    return n


def new_trust_workspace(layer: pvt_layer, k_max: int, device=None) -> torch.Tensor:
    ws = torch.empty(pvt_trust_workspace_bytes(layer, k_max), dtype=torch.uint8, device=device or "cuda")
    pvt_workspace_init(ws)
    return ws


def pvt_vstep_trust(layer: pvt_layer, k_max: int, ratio: float, idx_out: torch.Tensor, n_out: torch.Tensor,
                    stats_out: Optional[torch.Tensor], ws: torch.Tensor, stream=None) -> None:
    """V step with the subspace size taken from the trust ratio: idx_out (uint32 [k_max]) receives the groups in
    rank order, n_out (one int64/uint64) how many of them keep their new codes, stats_out (float64 [2] or None)
    the squared norm of the dequantised matrix before and the squared change that was kept."""
    _check(lib().pvt_vstep_trust(ctypes.byref(layer), k_max, ratio, idx_out.data_ptr(), n_out.data_ptr(),
                                 _ptr(stats_out), ws.data_ptr(), ws.numel() * ws.element_size(),
                                 _stream_ptr(stream)), "pvt_vstep_trust")


def pvt_vstep_refine(layer: pvt_layer, idx: torch.Tensor, k: int, max_moves: int,
                     err_out: Optional[torch.Tensor] = None, moves_out: Optional[torch.Tensor] = None,
                     status: Optional[torch.Tensor] = None, stream=None) -> None:
    """Local search over single-code changes (Appendix D) on the listed groups, from the stored codes."""
    _check(lib().pvt_vstep_refine(ctypes.byref(layer), idx.data_ptr(), k, max_moves, _ptr(err_out), _ptr(moves_out),
                                  _ptr(status), _stream_ptr(stream)), "pvt_vstep_refine")


def pvt_dequant(layer: pvt_layer, W_hat: torch.Tensor, status: Optional[torch.Tensor] = None, stream=None) -> None:
    _check(lib().pvt_dequant(ctypes.byref(layer), W_hat.data_ptr(), _OUT_DTYPE[W_hat.dtype], _ptr(status), _stream_ptr(stream)),
           "pvt_dequant")


_DTYPE = {torch.float32: PVT_F32, torch.float16: PVT_F16, torch.bfloat16: PVT_BF16}


_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream_for(device: int, stream, *tensors) -> int:
    """The stream's handle.  The calls enqueue on the current device: every tensor has to be there."""
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError("the tensors of a call lie on one CUDA device")
    if device < 0 or device != _current_device():
        raise ValueError(f"the tensors are on device {device}, not on the current CUDA device")
    return stream.cuda_stream if stream is not None else _raw_stream(device) if _raw_stream else _stream_ptr(None)


def _matrix(t: torch.Tensor, rows: int, cols: int, what: str):
    """(dtype, elements from row to row) of a matrix whose rows are contiguous."""
    dtype = _DTYPE.get(t.dtype)
    if dtype is None or t.shape != (rows, cols):
        raise ValueError(f"{what} has to be a float32, float16 or bfloat16 matrix of {rows} x {cols}")
    ld, step = t.stride()
    if cols > 1 and step != 1:
        raise ValueError(f"the rows of {what} have to be contiguous")
    if ld < cols:
        if rows > 1:
            raise ValueError(f"the rows of {what} overlap")
        ld = cols
    return dtype, ld


def _vector(t: Optional[torch.Tensor], n: int, dtype, what: str) -> Optional[int]:
    if t is None:
        return None
    if t.dtype != dtype or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{what} has to be {n} contiguous {dtype}")
    return t.data_ptr()


def _status_word(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is not None and (t.element_size() != 4 or t.numel() < 1):
        raise ValueError("status has to be a 4-byte integer")
    return _ptr(t)


# pvt_mx, pvt_distill and pvt_norm as bytes (a third of the time that a ctypes.Structure takes to make)
_pack_mx = struct.Struct("iiiiqPPP").pack
_pack_norm = struct.Struct("qiiPqPqPPiifi").pack
_pack_distill = struct.Struct("qiiPqifPPPP").pack


class Mx:
    """A matrix in 4-bit block floating point: its tensors and its descriptor (the bytes of a pvt_mx)."""

    def __init__(self, codes, scales, rows, cols, fmt, tensor_scale, ld, device):
        self.codes, self.scales, self.tensor_scale = codes, scales, tensor_scale
        self.rows, self.cols, self.format, self.device = rows, cols, fmt, device
        self.ref = _pack_mx(rows, cols, fmt, 0, ld, codes.data_ptr(), scales.data_ptr(),
                            0 if tensor_scale is None else tensor_scale.data_ptr())


def make_mx(codes: torch.Tensor, scales: torch.Tensor, rows: int, cols: int, fmt: int,
            tensor_scale: Optional[torch.Tensor] = None) -> Mx:
    """Describe a matrix whose arrays are CUDA tensors.  codes: uint8 [rows, at least ceil(cols / 2)], rows a multiple of 16
    bytes apart; scales: uint8, pvt_mx_scale_bytes of them; tensor_scale: one float32, for PVT_MX_E4M3_16 only."""
    shape = codes.shape
    if codes.dtype != torch.uint8 or len(shape) != 2 or shape[0] != rows or rows < 1 or cols < 1:
        raise ValueError("codes have to be uint8 [rows, bytes], rows and cols positive")
    # (a row is read in pieces of 16 bytes)
    ld, step = codes.stride()
    width = shape[1]
    if width % 16 or width < (cols + 31) // 32 * 16 or step != 1:
        raise ValueError("a row of codes has to be contiguous and hold ceil(cols / 32) * 16 bytes or a larger multiple of 16")
    if rows == 1:
        ld = width
    elif ld % 16 or ld < width:
        raise ValueError("rows of codes have to be a multiple of 16 bytes apart")
    if fmt not in (PVT_MX_E8M0_32, PVT_MX_E4M3_16):
        raise ValueError("unknown format")
    need = -(-rows // 128) * -(-cols // 256) * (1024 if fmt == PVT_MX_E8M0_32 else 2048)
    if scales.dtype != torch.uint8 or scales.numel() < need or not scales.is_contiguous():
        raise ValueError("scales have to be pvt_mx_scale_bytes contiguous uint8")
    device = codes.get_device()
    if tensor_scale is not None:
        if fmt != PVT_MX_E4M3_16 or tensor_scale.dtype != torch.float32 or tensor_scale.numel() != 1:
            raise ValueError("tensor_scale has to be one float32, for PVT_MX_E4M3_16")
        if tensor_scale.get_device() != device:
            raise ValueError("the tensors of a matrix lie on one CUDA device")
    if device < 0 or scales.get_device() != device:
        raise ValueError("the tensors of a matrix lie on one CUDA device")
    return Mx(codes, scales, rows, cols, fmt, tensor_scale, ld, device)


def new_mx(rows: int, cols: int, fmt: int, tensor_scale: Optional[torch.Tensor] = None, device=None) -> Mx:
    """Room for a matrix of that shape (its content is undefined until pvt_mx_quantize)."""
    device = device or "cuda"
    rows, cols = int(rows), int(cols)
    codes = torch.empty(rows, (cols + 31) // 32 * 16, dtype=torch.uint8, device=device)
    scales = torch.empty(pvt_mx_scale_bytes(rows, cols, fmt), dtype=torch.uint8, device=device)
    return make_mx(codes, scales, rows, cols, fmt, tensor_scale)


def pvt_mx_scale_bytes(rows: int, cols: int, fmt: int) -> int:
    n = int(lib().pvt_mx_scale_bytes(rows, cols, fmt))
    if n == 0:
        raise PvtError(PVT_EINVAL, "pvt_mx_scale_bytes")
    return n


def pvt_mx_quantize(m: Mx, x: torch.Tensor, stream=None) -> None:
    """x (float32, float16 or bfloat16 [rows, cols], rows of any distance) into m's codes and scales."""
    dtype, ld = _matrix(x, m.rows, m.cols, "x")
    _check(lib().pvt_mx_quantize(m.ref, x.data_ptr(), dtype, ld, _stream_for(m.device, stream, x)), "pvt_mx_quantize")


def pvt_mx_dequant(m: Mx, values: torch.Tensor, stream=None) -> None:
    """What m's codes and scales stand for."""
    dtype, ld = _matrix(values, m.rows, m.cols, "values")
    _check(lib().pvt_mx_dequant(m.ref, values.data_ptr(), dtype, ld, _stream_for(m.device, stream, values)),
           "pvt_mx_dequant")


def pvt_mx_product(x: Mx, w: Mx, y: torch.Tensor, status: Optional[torch.Tensor] = None, stream=None) -> None:
    """y [tokens, outputs] = x w^T on the block-scaled tensor cores; x [tokens, inputs], w [outputs, inputs]."""
    dtype, ld = _matrix(y, x.rows, w.rows, "y")
    _check(lib().pvt_mx_product(x.ref, w.ref, y.data_ptr(), dtype, ld, _status_word(status),
                                _stream_for(x.device, stream, w.codes, y, status)), "pvt_mx_product")


def _gradient(dy: torch.Tensor, tokens: int, outputs: int) -> int:
    """Elements from row to row of the gradient of a product's result."""
    dtype, ld = _matrix(dy, tokens, outputs, "dy")
    if dtype != PVT_BF16:
        raise ValueError("dy has to be bfloat16")
    return (ld + 7) // 8 * 8 if tokens == 1 else ld


def pvt_mx_grad_input(dy: torch.Tensor, w: Mx, dx: torch.Tensor, status: Optional[torch.Tensor] = None, stream=None) -> None:
    """dx [tokens, inputs] = dy w; dy bfloat16 [tokens, outputs], 16-byte aligned, rows a multiple of 8 elements apart."""
    ldy = _gradient(dy, dy.shape[0], w.rows)
    dtype, ld = _matrix(dx, dy.shape[0], w.cols, "dx")
    _check(lib().pvt_mx_grad_input(dy.data_ptr(), ldy, dy.shape[0], w.ref, dx.data_ptr(), dtype, ld, _status_word(status),
                                   _stream_for(w.device, stream, dy, dx, status)), "pvt_mx_grad_input")


def pvt_mx_grad_weight(dy: torch.Tensor, x: Mx, dw: torch.Tensor, accumulate: bool = False,
                       status: Optional[torch.Tensor] = None, stream=None) -> None:
    """dw [outputs, inputs] (float32) = dy^T x, added to what it holds if accumulate; dy as for pvt_mx_grad_input."""
    ldy = _gradient(dy, x.rows, dy.shape[1])
    dtype, ld = _matrix(dw, dy.shape[1], x.cols, "dw")
    if dtype != PVT_F32:
        raise ValueError("dw has to be float32")
    _check(lib().pvt_mx_grad_weight(dy.data_ptr(), ldy, dy.shape[1], x.ref, dw.data_ptr(), ld, 1 if accumulate else 0,
                                    _status_word(status), _stream_for(x.device, stream, dy, dw, status)),
           "pvt_mx_grad_weight")


def pvt_mx_gated(x: Mx, w_gate: Mx, w_up: Mx, h: Optional[torch.Tensor] = None, quantized: Optional[Mx] = None,
                 activation: int = PVT_ACT_SILU, status: Optional[torch.Tensor] = None, stream=None) -> None:
    """h [tokens, outputs] = f(x w_gate^T) (x w_up^T), of any type, and / or the same as a 4-bit matrix of x's format."""
    ptr, dtype, ld, ref = None, PVT_F32, 0, None
    if h is not None:
        dtype, ld = _matrix(h, x.rows, w_gate.rows, "h")
        ptr = h.data_ptr()
    if quantized is not None:
        if quantized.rows != x.rows or quantized.cols != w_gate.rows or quantized.format != x.format:
            raise ValueError("quantized has to be tokens x outputs, of x's format")
        ref = quantized.ref
    _check(lib().pvt_mx_gated(x.ref, w_gate.ref, w_up.ref, activation, ptr, dtype, ld, ref, _status_word(status),
                              _stream_for(x.device, stream, w_gate.codes, w_up.codes, h, quantized and quantized.codes, status)),
           "pvt_mx_gated")


def pvt_mx_gated_grad(x: Mx, w_gate: Mx, w_up: Mx, dh: torch.Tensor, dgate: torch.Tensor, dup: torch.Tensor,
                      activation: int = PVT_ACT_SILU, status: Optional[torch.Tensor] = None, stream=None) -> None:
    """dgate and dup, bfloat16 [tokens, outputs] as pvt_mx_grad_weight takes them, from dh (any type; either may be dh itself)."""
    dtype, ldh = _matrix(dh, x.rows, w_gate.rows, "dh")
    ldd = _gradient_pair(dgate, dup, x.rows, w_gate.rows)
    _check(lib().pvt_mx_gated_grad(x.ref, w_gate.ref, w_up.ref, activation, dh.data_ptr(), dtype, ldh, dgate.data_ptr(),
                                   dup.data_ptr(), ldd, _status_word(status),
                                   _stream_for(x.device, stream, w_gate.codes, w_up.codes, dh, dgate, dup, status)), "pvt_mx_gated_grad")


def _gradient_pair(dgate: torch.Tensor, dup: torch.Tensor, tokens: int, outputs: int) -> int:
    ldd, other = _gradient(dgate, tokens, outputs), _gradient(dup, tokens, outputs)
    if tokens > 1 and ldd != other:
        raise ValueError("the rows of dgate and dup have to be equally far apart")
    return min(ldd, other)


def pvt_mx_gated_grad_input(dgate: torch.Tensor, dup: torch.Tensor, w_gate: Mx, w_up: Mx, dx: torch.Tensor,
                            status: Optional[torch.Tensor] = None, stream=None) -> None:
    """dx [tokens, inputs] = dgate w_gate + dup w_up; the two matrices share their tensor_scale, if they have one."""
    tokens = dgate.shape[0]
    ldd = _gradient_pair(dgate, dup, tokens, w_gate.rows)
    dtype, ld = _matrix(dx, tokens, w_gate.cols, "dx")
    _check(lib().pvt_mx_gated_grad_input(dgate.data_ptr(), dup.data_ptr(), ldd, tokens, w_gate.ref, w_up.ref, dx.data_ptr(), dtype, ld,
                                         _status_word(status), _stream_for(w_gate.device, stream, w_up.codes, dgate, dup, dx, status)),
           "pvt_mx_gated_grad_input")


def pvt_distill_top(logits: torch.Tensor, top_idx: torch.Tensor, top_logit: torch.Tensor, lse: Optional[torch.Tensor] = None,
                    temperature: float = 1.0, stream=None) -> None:
    """The k largest logits of each row (int32 and float32 [rows, k], in order) and log sum exp(logits / temperature)."""
    rows, vocab = logits.shape
    dtype, ld = _matrix(logits, rows, vocab, "logits")
    k = int(top_idx.shape[-1])
    idx, val = _vector(top_idx, rows * k, torch.int32, "top_idx"), _vector(top_logit, rows * k, torch.float32, "top_logit")
    out = _vector(lse, rows, torch.float32, "lse")
    _check(lib().pvt_distill_top(logits.data_ptr(), dtype, ld, rows, vocab, k, temperature, idx, val, out,
                                 _stream_for(logits.get_device(), stream, top_idx, top_logit, lse)), "pvt_distill_top")


class Distill:
    """The student's logits and what they are trained against: the tensors and their descriptor."""

    def __init__(self, ref, tensors, rows, vocab, device):
        self.ref, self.tensors = ref, tensors  # (the bytes of a pvt_distill)
        self.device, self.rows, self.vocab = device, rows, vocab


def make_distill(logits: torch.Tensor, top_idx: torch.Tensor, top_logit: torch.Tensor,
                 teacher_lse: Optional[torch.Tensor] = None, weight: Optional[torch.Tensor] = None,
                 temperature: float = 1.0) -> Distill:
    """logits [rows, vocab] against the teacher's list (int32 and float32 [rows, k]).  With teacher_lse (float32 [rows], of the
    same temperature) everything that is not listed is one more outcome, without it the listed probabilities add up to 1.  A list
    that names everything the teacher's mask leaves has no rest (include/pvt.h says when what rounding leaves is taken for none)."""
    rows, vocab = logits.shape
    dtype, ld = _matrix(logits, rows, vocab, "logits")
    k = int(top_idx.shape[-1])
    ref = _pack_distill(rows, vocab, k, logits.data_ptr(), ld, dtype, float(temperature),
                        _vector(top_idx, rows * k, torch.int32, "top_idx"),
                        _vector(top_logit, rows * k, torch.float32, "top_logit"),
                        _vector(teacher_lse, rows, torch.float32, "teacher_lse") or 0,
                        _vector(weight, rows, torch.float32, "weight") or 0)
    tensors = (logits, top_idx, top_logit, teacher_lse, weight)
    device = logits.get_device()
    for t in tensors:
        if t is not None and (device < 0 or t.get_device() != device):
            raise ValueError("the tensors of a distillation lie on one CUDA device")
    return Distill(ref, tensors, rows, vocab, device)


def pvt_distill_loss(d: Distill, loss: torch.Tensor, stats: Optional[torch.Tensor] = None,
                     upstream: Optional[torch.Tensor] = None, grad: Optional[torch.Tensor] = None,
                     status: Optional[torch.Tensor] = None, stream=None) -> None:
    """loss (float32 [rows]); with grad ([rows, vocab], may be the logits) the gradient in the same pass, with stats (float32
    [rows, PVT_DISTILL_STATS]) what pvt_distill_grad needs."""
    dtype, ld = _matrix(grad, d.rows, d.vocab, "grad") if grad is not None else (PVT_F32, 0)
    out = _vector(loss, d.rows, torch.float32, "loss")
    st = _vector(stats, d.rows * PVT_DISTILL_STATS, torch.float32, "stats")
    up = _vector(upstream, d.rows, torch.float32, "upstream")
    _check(lib().pvt_distill_loss(d.ref, out, st, up, _ptr(grad), dtype, ld, _status_word(status),
                                  _stream_for(d.device, stream, loss, stats, upstream, grad, status)), "pvt_distill_loss")


def pvt_distill_grad(d: Distill, stats: torch.Tensor, grad: torch.Tensor, upstream: Optional[torch.Tensor] = None,
                     status: Optional[torch.Tensor] = None, stream=None) -> None:
    """The gradient from the statistics of an earlier pvt_distill_loss on the same d."""
    dtype, ld = _matrix(grad, d.rows, d.vocab, "grad")
    st = _vector(stats, d.rows * PVT_DISTILL_STATS, torch.float32, "stats")
    up = _vector(upstream, d.rows, torch.float32, "upstream")
    _check(lib().pvt_distill_grad(d.ref, st, up, grad.data_ptr(), dtype, ld, _status_word(status),
                                  _stream_for(d.device, stream, stats, upstream, grad, status)), "pvt_distill_grad")


class Norm:
    """Rows to be normalised, their weights, and the descriptor (the bytes of a pvt_norm)."""

    def __init__(self, ref, tensors, rows, cols, dtype, device):
        self.ref, self.tensors = ref, tensors
        self.device, self.rows, self.cols, self.dtype = device, rows, cols, dtype


def make_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, *,
              kind: int = PVT_NORM_LAYER, eps: float = 1e-5, residual: Optional[torch.Tensor] = None) -> Norm:
    """Describe the norm of the rows of x + residual (float32, float16 or bfloat16 [rows, cols], one type, rows of any distance);
    weight and bias [cols], contiguous, of any of these types, both the same.  For pvt_norm_grad x is the sum and there is no residual."""
    if x.dim() != 2:
        raise ValueError("x has to be a matrix")
    rows, cols = x.shape
    dtype, ld = _matrix(x, rows, cols, "x")
    res, ldr = 0, 0
    if residual is not None:
        other, ldr = _matrix(residual, rows, cols, "residual")
        if other != dtype:
            raise ValueError("residual has to be of x's type")
        res = residual.data_ptr()
    w_type = (weight if weight is not None else bias).dtype if weight is not None or bias is not None else torch.float32
    if w_type not in _DTYPE:
        raise ValueError("weight and bias have to be float32, float16 or bfloat16")
    device = x.get_device()
    for t in (x, residual, weight, bias):
        if t is not None and (device < 0 or t.get_device() != device):
            raise ValueError("the tensors of a norm lie on one CUDA device")
    ref = _pack_norm(rows, cols, kind, x.data_ptr(), ld, res, ldr, _vector(weight, cols, w_type, "weight") or 0,
                     _vector(bias, cols, w_type, "bias") or 0, dtype, _DTYPE[w_type], eps, 0)
    return Norm(ref, (x, residual, weight, bias), rows, cols, dtype, device)


def pvt_norm_apply(n: Norm, y: Optional[torch.Tensor] = None, quantized: Optional[Mx] = None, total: Optional[torch.Tensor] = None,
                   stats: Optional[torch.Tensor] = None, stream=None) -> None:
    """y [rows, cols] of any type, and / or the same as a 4-bit matrix; total: x + residual, of their type (may be either of
    them); stats: float32 [rows, 2], mean and 1 / deviation of each row, for pvt_norm_grad."""
    t_ptr, ldt, y_ptr, y_dtype, ldy, q_ref = None, 0, None, PVT_F32, 0, None
    if total is not None:
        t_dtype, ldt = _matrix(total, n.rows, n.cols, "total")
        if t_dtype != n.dtype:
            raise ValueError("total has to be of x's type")
        t_ptr = total.data_ptr()
    if y is not None:
        y_dtype, ldy = _matrix(y, n.rows, n.cols, "y")
        y_ptr = y.data_ptr()
    if quantized is not None:
        if quantized.rows != n.rows or quantized.cols != n.cols:
            raise ValueError("quantized has to be of x's shape")
        q_ref = quantized.ref
    st = _vector(stats, 2 * n.rows, torch.float32, "stats")
    _check(lib().pvt_norm_apply(n.ref, t_ptr, ldt, y_ptr, y_dtype, ldy, q_ref, st,
                                _stream_for(n.device, stream, total, y, quantized and quantized.codes, stats)), "pvt_norm_apply")


def pvt_norm_workspace_bytes(n: Norm) -> int:
    return int(lib().pvt_norm_workspace_bytes(n.ref))


def new_norm_workspace(n: Norm, any_rows: bool = False) -> torch.Tensor:
    """Workspace for pvt_norm_grad with weights' gradients; it may be kept for further calls on as many rows and columns, or with
    any_rows for any number of rows (what is needed grows with them up to a few for each block that the GPU runs at once)."""
    ref = bytes(pvt_norm(rows=2 ** 31 - 1, cols=n.cols)) if any_rows else n.ref
    return torch.empty(int(lib().pvt_norm_workspace_bytes(ref)), dtype=torch.uint8, device=torch.device("cuda", n.device))


def pvt_norm_grad(n: Norm, stats: torch.Tensor, dy: torch.Tensor, dx: torch.Tensor, dresidual: Optional[torch.Tensor] = None,
                  dweight: Optional[torch.Tensor] = None, dbias: Optional[torch.Tensor] = None, accumulate: bool = False,
                  workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """dx [rows, cols] from dy and, if given, dresidual (one type; dx may be either of them or x); dweight and dbias [cols], float32, or
    float64 as pvt_adam_update takes them, added to what they hold if accumulate."""
    dtype, ldy = _matrix(dy, n.rows, n.cols, "dy")
    x_dtype, ldx = _matrix(dx, n.rows, n.cols, "dx")
    r_dtype, ldr = _matrix(dresidual, n.rows, n.cols, "dresidual") if dresidual is not None else (dtype, 0)
    if x_dtype != dtype or r_dtype != dtype:
        raise ValueError("dy, dx and dresidual have to be of one type")
    w_type = (dweight if dweight is not None else dbias).dtype if dweight is not None or dbias is not None else torch.float32
    if w_type not in (torch.float32, torch.float64):
        raise ValueError("dweight and dbias have to be float32 or float64")
    dw, db = _vector(dweight, n.cols, w_type, "dweight"), _vector(dbias, n.cols, w_type, "dbias")
    st = _vector(stats, 2 * n.rows, torch.float32, "stats")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().pvt_norm_grad(n.ref, st, dtype, dy.data_ptr(), ldy, _ptr(dresidual), ldr, dx.data_ptr(), ldx, dw, db,
                               PVT_F64 if w_type == torch.float64 else PVT_F32, 1 if accumulate else 0, _ptr(workspace), ws_bytes,
                               _stream_for(n.device, stream, stats, dy, dx, dresidual, dweight, dbias, workspace)), "pvt_norm_grad")


class Block:
    """Host arrays for pvt_vstep_block: the layers of one model block, their subspace sizes and output pointers
    (marshalled once; the tensors must stay alive while the block is used)."""

    def __init__(self, layers, ks, idx_outs, W_hats=None):
        n = len(layers)
        self.n = n
        self.layers = (pvt_layer * n)(*layers)
        self.k = (ctypes.c_uint64 * n)(*[int(x) for x in ks])
        self.idx = (ctypes.c_void_p * n)(*[t.data_ptr() for t in idx_outs])
        self.W_hat = None
        self.out_dtype = PVT_F32
        if W_hats is not None:
            self.W_hat = (ctypes.c_void_p * n)(*[None if t is None else t.data_ptr() for t in W_hats])
            dts = {t.dtype for t in W_hats if t is not None}
            if len(dts) > 1:
                raise ValueError("the dequantised matrices of a block share one dtype")
            if dts:
                self.out_dtype = _OUT_DTYPE[dts.pop()]
        self._keep = (list(idx_outs), list(W_hats) if W_hats is not None else None)

    def workspace_bytes(self) -> int:
        need = int(lib().pvt_block_workspace_bytes(self.layers, self.k, self.n))
        if need == 0:
            raise PvtError(PVT_EINVAL, "pvt_block_workspace_bytes")
        return need


class OneLayer:
    """pvt_vstep_block for one layer: the call's one-entry host arrays."""

    def __init__(self):
        self._k = (ctypes.c_uint64 * 1)()
        self._idx = (ctypes.c_void_p * 1)()
        self._W_hat = (ctypes.c_void_p * 1)()

    def step(self, layer: pvt_layer, k: int, idx_out: torch.Tensor, W_hat: Optional[torch.Tensor], ws: torch.Tensor,
             stream=None) -> None:
        """select -> encode -> dequantise (the last if W_hat is given), one C call."""
        self._k[0] = k
        self._idx[0] = idx_out.data_ptr()
        out, dtype = None, PVT_F32
        if W_hat is not None:
            self._W_hat[0] = W_hat.data_ptr()
            out, dtype = self._W_hat, _OUT_DTYPE[W_hat.dtype]
        _check(lib().pvt_vstep_block(ctypes.byref(layer), self._k, 1, self._idx, out, dtype, ws.data_ptr(),
                                     ws.numel() * ws.element_size(), _stream_ptr(stream)), "pvt_vstep_block")


def pvt_vstep_block(block: Block, ws: torch.Tensor, stream=None) -> None:
    """select -> encode -> dequantise over every layer of the block, one C call."""
    _check(lib().pvt_vstep_block(block.layers, block.k, block.n, block.idx, block.W_hat, block.out_dtype, ws.data_ptr(),
                                 ws.numel() * ws.element_size(), _stream_ptr(stream)), "pvt_vstep_block")


def pvt_pstep_grad(layer: pvt_layer, grad_codebooks: torch.Tensor, grad_scale: Optional[torch.Tensor] = None,
                   status: Optional[torch.Tensor] = None, stream=None) -> None:
    """grad_codebooks [M, K, 8] float64, grad_scale [rows] float64 or None (both overwritten)."""
    assert grad_codebooks.dtype == torch.float64 and (grad_scale is None or grad_scale.dtype == torch.float64)
    _check(lib().pvt_pstep_grad(ctypes.byref(layer), grad_codebooks.data_ptr(), _ptr(grad_scale), _ptr(status),
                                _stream_ptr(stream)), "pvt_pstep_grad")


def pvt_adam_bias(step: int, beta1: float, beta2: float):
    """Bias corrections 1 - beta^t of step t >= 1 as the binary32 numbers pvt_adam_update takes."""
    b1, b2 = ctypes.c_float(0.0), ctypes.c_float(0.0)
    _check(lib().pvt_adam_bias(step, beta1, beta2, ctypes.byref(b1), ctypes.byref(b2)), "pvt_adam_bias")
    return b1.value, b2.value


def pvt_adam_update(param: torch.Tensor, grad: torch.Tensor, exp_avg: torch.Tensor, exp_avg_sq: torch.Tensor,
                    step: int, lr: float, beta1: float = 0.9, beta2: float = 0.95, eps: float = 1e-8,
                    param_f16: Optional[torch.Tensor] = None, stream=None) -> None:
    """One Adam update in place (param, exp_avg, exp_avg_sq float32; grad float64; optional float16 copy)."""
    assert param.dtype == torch.float32 and grad.dtype == torch.float64
    assert exp_avg.dtype == torch.float32 and exp_avg_sq.dtype == torch.float32
    assert param_f16 is None or param_f16.dtype == torch.float16
    bias1, bias2 = pvt_adam_bias(step, beta1, beta2)
    _check(lib().pvt_adam_update(param.data_ptr(), _ptr(param_f16), grad.data_ptr(), exp_avg.data_ptr(),
                                 exp_avg_sq.data_ptr(), param.numel(), lr, beta1, beta2, eps, bias1, bias2,
                                 _stream_ptr(stream)), "pvt_adam_update")


def pvt_adam_direction(grad: torch.Tensor, exp_avg: torch.Tensor, exp_avg_sq: torch.Tensor, out: torch.Tensor,
                       step: int, beta1: float = 0.9, beta2: float = 0.95, eps: float = 1e-8, stream=None) -> None:
    """Adam-normalised update direction of the V step (all float32; moments updated in place)."""
    for t in (grad, exp_avg, exp_avg_sq, out):
        assert t.dtype == torch.float32 and t.is_contiguous()
    bias1, bias2 = pvt_adam_bias(step, beta1, beta2)
    _check(lib().pvt_adam_direction(grad.data_ptr(), exp_avg.data_ptr(), exp_avg_sq.data_ptr(), out.data_ptr(),
                                    grad.numel(), beta1, beta2, eps, bias1, bias2, _stream_ptr(stream)),
           "pvt_adam_direction")


def pvt_status(ws: torch.Tensor, stream=None) -> int:
    rc = int(lib().pvt_status(ws.data_ptr(), _stream_ptr(stream)))
    if rc < 0:
        raise PvtError(rc, "pvt_status")
    return rc


def pvt_version() -> int:
    return int(lib().pvt_version())


def pvt_set_m1_search(mode: int) -> None:
    """Engine of the single-codebook search: PVT_M1_AUTO, PVT_M1_FP32 or PVT_M1_TENSOR."""
    lib().pvt_set_m1_search(mode)


def pvt_probe_fp32_tflops(stream=None) -> float:
    """Measured FP32 FMA throughput of the current device in TFLOP/s (a short kernel of independent FMA chains)."""
    props = torch.cuda.get_device_properties(torch.cuda.current_device())
    scratch = torch.empty(props.multi_processor_count * 2048, dtype=torch.float32, device="cuda")
    out = ctypes.c_float(0.0)
    _check(lib().pvt_probe_fp32_tflops(scratch.data_ptr(), scratch.numel(), ctypes.byref(out), _stream_ptr(stream)),
           "pvt_probe_fp32_tflops")
    return float(out.value)


def pvt_test_wait_limit(max_polls: int = 0, withhold_copy: int = -1) -> None:
    """Test hook: poll limit of the search kernels' on-chip waits (0 = default) and the sequence number of a
    codebook copy that every thread block leaves out (-1 = none).  Process-wide."""
    lib().pvt_test_wait_limit(max_polls, withhold_copy)


def pvt_launch_count() -> int:
    return int(lib().pvt_launch_count())


def pvt_timing_enable(on: bool) -> None:
    lib().pvt_timing_enable(1 if on else 0)


def pvt_timing_read(kernel_id: int):
    """(total milliseconds, launches) of one kernel class since the last read."""
    ms, n = ctypes.c_float(0.0), ctypes.c_int(0)
    _check(lib().pvt_timing_read(kernel_id, ctypes.byref(ms), ctypes.byref(n)), "pvt_timing_read")
    return float(ms.value), int(n.value)


def pvt_evaluated_share(layer: pvt_layer, k: int, ws: torch.Tensor) -> float:
    """Share of the (target, codeword) pairs that the search of k groups which used the workspace last has evaluated; waits
    for it."""
    at = int(lib().pvt_search_counts(ctypes.byref(layer), k))
    if at == 0:
        return 1.0
    tiles, steps = -(-k // 256), -(-layer.codebook_size // 128)
    beyond = int(ws[at:at + 4 * tiles].view(torch.int32).sum())
    return (beyond + 32 * tiles) / (tiles * steps)
