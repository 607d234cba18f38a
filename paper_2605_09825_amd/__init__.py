"""Python binding of libmxfp4.so (the gfx950 MXFP4 linear-layer library).

Argument marshalling only: every function here forwards to the C-ABI entry point
of the same name (include/mxfp4.h) with raw device pointers and the current torch
stream; torch is used for device memory and streams and for nothing else.  There is
no fallback: if the HIP library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Tuple

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libmxfp4.so")
if os.environ.get("MXFP4_SANITIZE_HOST", "") not in ("", "0"):  # host-sanitizer build (see build.py)
    LIB_PATH = os.path.join(HERE, "libmxfp4_san.so")

# enums of include/mxfp4.h
OK, EINVAL, ESHAPE, EALIGN, EWORKSPACE, EDEVICE, ENOTIMPL = range(7)
AXIS_LAST, AXIS_FIRST = 0, 1
HAD_NONE, HAD_DET, HAD_RANDSIGN, HAD_DET16, HAD_RANDSIGN16 = 0, 1, 2, 3, 4
RNE, SR = 0, 1
OUT_BF16, OUT_FP32 = 0, 1
GEOM_1D, GEOM_2D = 0, 1
FMT_E2M1, FMT_E4M3 = 0, 1
ROPE_HALF, ROPE_PAIRS = 0, 1
ROPE_SCALE_NONE, ROPE_SCALE_LINEAR, ROPE_SCALE_NTK, ROPE_SCALE_YARN, ROPE_SCALE_WAVELENGTH = range(5)

EXPORTS = ("mxfp4_quantize", "mxfp4_quantize_dual", "mxfp4_quantize_2d", "mxfp4_quantize_fp8",
           "mxfp4_quantize_fp8_dual", "mxfp4_gemm",
           "mxfp4_gemm_fmt", "mxfp4_gemm_pair", "mxfp4_gemm_plan", "mxfp4_gemm_route",
           "mxfp4_gemm_pair_route", "mxfp4_linear_fwd", "mxfp4_linear_fwd_static", "mxfp4_linear_bwd",
           "mxfp4_linear_fwd_save", "mxfp4_linear_bwd_saved", "mxfp4_linear_saved_bytes",
           "mxfp4_linear_saved_layout", "mxfp4_linear_workspace_bytes", "mxfp4_linear_workspace_layout",
           "mxfp4_residual_norm_fwd", "mxfp4_residual_norm_bwd", "mxfp4_residual_norm_workspace_bytes", "mxfp4_rope_table", "mxfp4_rope",
           "mxfp4_orthogonalize", "mxfp4_orthogonalize_workspace_bytes",
           "mxfp4_status_string")


class LinearCfg(ctypes.Structure):
    """mxfp4_linear_cfg"""
    _fields_ = [("hadamard", ctypes.c_int32), ("rounding", ctypes.c_int32), ("seed", ctypes.c_uint64),
                ("y_dtype", ctypes.c_int32), ("dx_dtype", ctypes.c_int32), ("dw_dtype", ctypes.c_int32),
                ("dw_accumulate", ctypes.c_int32), ("geometry", ctypes.c_int32), ("fprop_format", ctypes.c_int32),
                ("dgrad_format", ctypes.c_int32), ("wgrad_format", ctypes.c_int32)]


class NormCfg(ctypes.Structure):
    """mxfp4_norm_cfg"""
    _fields_ = [("eps", ctypes.c_float), ("residual_scale", ctypes.c_float), ("branch_scale", ctypes.c_float),
                ("weight_offset", ctypes.c_float), ("post_norm", ctypes.c_int32), ("accumulate", ctypes.c_int32)]


class RopeCfg(ctypes.Structure):
    """mxfp4_rope_cfg"""
    _fields_ = [("base", ctypes.c_double), ("factor", ctypes.c_double), ("low", ctypes.c_double), ("high", ctypes.c_double),
                ("original_positions", ctypes.c_double), ("attention_factor", ctypes.c_double), ("scaling", ctypes.c_int32)]


class MuonCfg(ctypes.Structure):
    """mxfp4_muon_cfg"""
    _fields_ = [("momentum", ctypes.c_float), ("nesterov", ctypes.c_int32), ("steps", ctypes.c_int32), ("a", ctypes.c_float),
                ("b", ctypes.c_float), ("c", ctypes.c_float), ("eps", ctypes.c_float), ("out_scale", ctypes.c_float), ("join_steps", ctypes.c_int32)]


class Mxfp4Error(RuntimeError):
    def __init__(self, call: str, status: int):
        self.status = status
        super().__init__(f"{call} failed: status {status} ({status_string(status)})")


_lib: Optional[ctypes.CDLL] = None


def lib() -> ctypes.CDLL:
    """Load libmxfp4.so (built by paper_2605_09825_amd.build); raises if it is not there."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2605_09825_amd.build` (there is no CPU fallback)")
        L = ctypes.CDLL(LIB_PATH)
        vp, i64, ci, u64, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_uint64, ctypes.c_size_t
        L.mxfp4_quantize.restype = ci
        L.mxfp4_quantize.argtypes = [vp, i64, i64, i64, ci, ci, ci, u64, vp, vp, vp]
        L.mxfp4_quantize_dual.restype = ci
        L.mxfp4_quantize_dual.argtypes = [vp, i64, i64, i64, ci, ci, u64, vp, vp, vp, vp, vp]
        L.mxfp4_quantize_fp8.restype = ci
        L.mxfp4_quantize_fp8.argtypes = [vp, i64, i64, i64, ci, ci, u64, vp, vp, vp]
        L.mxfp4_quantize_fp8_dual.restype = ci
        L.mxfp4_quantize_fp8_dual.argtypes = [vp, i64, i64, i64, ci, u64, vp, vp, vp, vp, vp]
        L.mxfp4_gemm_fmt.restype = ci
        L.mxfp4_gemm_fmt.argtypes = [vp, vp, ci, vp, vp, ci, i64, i64, i64, vp, i64, ci, ci, vp]
        L.mxfp4_quantize_2d.restype = ci
        L.mxfp4_quantize_2d.argtypes = [vp, i64, i64, i64, ci, ci, u64, vp, vp, vp, vp, vp]
        L.mxfp4_linear_fwd_save.restype = ci
        L.mxfp4_linear_fwd_save.argtypes = [vp, vp, vp, i64, i64, i64, ctypes.POINTER(LinearCfg), vp, sz, vp, sz, vp]
        L.mxfp4_linear_bwd_saved.restype = ci
        L.mxfp4_linear_bwd_saved.argtypes = [vp, vp, sz, vp, vp, i64, i64, i64, ctypes.POINTER(LinearCfg), vp, sz, vp]
        L.mxfp4_linear_saved_bytes.restype = sz
        L.mxfp4_linear_saved_bytes.argtypes = [i64, i64, i64, ctypes.POINTER(LinearCfg)]
        L.mxfp4_linear_saved_layout.restype = ci
        L.mxfp4_linear_saved_layout.argtypes = [i64, i64, i64, ctypes.POINTER(LinearCfg), ctypes.POINTER(sz)]
        L.mxfp4_gemm.restype = ci
        L.mxfp4_gemm.argtypes = [vp, vp, vp, vp, i64, i64, i64, vp, i64, ci, ci, vp]
        L.mxfp4_linear_fwd.restype = ci
        L.mxfp4_linear_fwd.argtypes = [vp, vp, vp, i64, i64, i64, ctypes.POINTER(LinearCfg), vp, sz, vp]
        L.mxfp4_gemm_pair.restype = ci
        L.mxfp4_gemm_pair.argtypes = ([vp, vp, vp, vp, i64, i64, i64, vp, i64, ci] +
                                      [vp, vp, vp, vp, i64, i64, i64, vp, i64, ci, ci] + [vp])
        L.mxfp4_gemm_plan.restype = ci
        L.mxfp4_gemm_plan.argtypes = [i64, i64, i64, ci, ci, i64, ci, ctypes.POINTER(ci), ctypes.POINTER(i64)]
        L.mxfp4_gemm_route.restype = ci
        L.mxfp4_gemm_route.argtypes = [i64, i64, i64, ci, ci, i64, ci, ci, ci, ctypes.POINTER(ci)]
        L.mxfp4_gemm_pair_route.restype = ci
        L.mxfp4_gemm_pair_route.argtypes = ([i64, i64, i64, ci, i64, ci] * 2) + [ci, ci, ctypes.POINTER(ci)]
        L.mxfp4_linear_fwd_static.restype = ci
        L.mxfp4_linear_fwd_static.argtypes = [vp, vp, vp, i64, i64, i64, ctypes.POINTER(LinearCfg), vp]
        L.mxfp4_linear_bwd.restype = ci
        L.mxfp4_linear_bwd.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, ctypes.POINTER(LinearCfg), vp, sz, vp]
        L.mxfp4_linear_workspace_bytes.restype = sz
        L.mxfp4_linear_workspace_bytes.argtypes = [i64, i64, i64, ctypes.POINTER(LinearCfg), ci]
        L.mxfp4_linear_workspace_layout.restype = ci
        L.mxfp4_linear_workspace_layout.argtypes = [i64, i64, i64, ctypes.POINTER(LinearCfg), ci, ctypes.POINTER(sz)]
        L.mxfp4_residual_norm_fwd.restype = ci
        L.mxfp4_residual_norm_fwd.argtypes = [vp, i64, vp, i64, vp, i64, vp, vp, i64, i64, ci, ci, ctypes.POINTER(NormCfg), vp, i64,
                                              vp, i64, vp, vp]
        L.mxfp4_residual_norm_bwd.restype = ci
        L.mxfp4_residual_norm_bwd.argtypes = [vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, vp, i64, i64, ci, ci,
                                              ctypes.POINTER(NormCfg), vp, i64, vp, i64, vp, i64, vp, vp, vp, sz, vp]
        L.mxfp4_residual_norm_workspace_bytes.restype = sz
        L.mxfp4_residual_norm_workspace_bytes.argtypes = [i64, i64]
        L.mxfp4_rope_table.restype = ci
        L.mxfp4_rope_table.argtypes = [vp, i64, i64, ctypes.POINTER(RopeCfg), vp]
        L.mxfp4_rope.restype = ci
        L.mxfp4_rope.argtypes = [vp, i64, i64, vp, i64, i64, i64, i64, i64, i64, ci, ci, ci, vp, i64, vp, i64, vp]
        L.mxfp4_orthogonalize.restype = ci
        L.mxfp4_orthogonalize.argtypes = [vp, i64, i64, vp, vp, i64, i64, i64, i64, i64, ci, ctypes.POINTER(MuonCfg), vp, sz, vp]
        L.mxfp4_orthogonalize_workspace_bytes.restype = sz
        L.mxfp4_orthogonalize_workspace_bytes.argtypes = [i64, i64, i64]
        L.mxfp4_status_string.restype = ctypes.c_char_p
        L.mxfp4_status_string.argtypes = [ci]
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().mxfp4_status_string(int(status)).decode()


def _check(call: str, status: int) -> None:
    if status != OK:
        raise Mxfp4Error(call, status)


def _stream_ptr(stream) -> int:
    # (the handle of the current device's current stream, without the Stream object that torch.cuda.current_stream()
    # builds around it: 2.9 us of the 8 us that a call of a small product took on the host)
    if stream is not None:
        return int(stream.cuda_stream)
    import torch
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _ptr(t) -> Optional[int]:
    return None if t is None else int(t.data_ptr())


def _out_dtype(code: int):
    import torch
    return torch.float32 if code == OUT_FP32 else torch.bfloat16


# ---------------------------------------------------------------------------------------
def mxfp4_quantize(x, axis: int = AXIS_LAST, hadamard: int = HAD_NONE, rounding: int = RNE, seed: int = 0,
                   q=None, s=None, stream=None) -> Tuple["torch.Tensor", "torch.Tensor"]:
    """x: bf16 CUDA tensor [rows][cols] with unit inner stride.  Returns (q, s) uint8 tensors
    [R][C/2] and [R][C/32] (allocated here with torch.empty unless passed in)."""
    import torch
    assert x.is_cuda and x.dtype == torch.bfloat16 and x.dim() == 2 and (x.numel() == 0 or x.stride(1) == 1)
    rows, cols = x.shape
    ld = x.stride(0) if rows > 1 else max(cols, x.stride(0))
    R, C = (rows, cols) if axis == AXIS_LAST else (cols, rows)
    if q is None:
        q = torch.empty((R, C // 2), dtype=torch.uint8, device=x.device)
    if s is None:
        s = torch.empty((R, C // 32), dtype=torch.uint8, device=x.device)
    _check("mxfp4_quantize", lib().mxfp4_quantize(_ptr(x), rows, cols, ld, axis, hadamard, rounding,
                                                  seed & (2**64 - 1), _ptr(q), _ptr(s), _stream_ptr(stream)))
    return q, s


def mxfp4_quantize_dual(x, hadamard: int = HAD_NONE, rounding: int = RNE, seed: int = 0, stream=None):
    """Both quantisations of x [rows][cols] from one pass: returns (q_last, s_last, q_first, s_first)."""
    import torch
    assert x.is_cuda and x.dtype == torch.bfloat16 and x.dim() == 2 and (x.numel() == 0 or x.stride(1) == 1)
    rows, cols = x.shape
    ld = x.stride(0) if rows > 1 else max(cols, x.stride(0))
    u8 = dict(dtype=torch.uint8, device=x.device)
    ql, sl = torch.empty((rows, cols // 2), **u8), torch.empty((rows, cols // 32), **u8)
    qf, sf = torch.empty((cols, rows // 2), **u8), torch.empty((cols, rows // 32), **u8)
    _check("mxfp4_quantize_dual", lib().mxfp4_quantize_dual(_ptr(x), rows, cols, ld, hadamard, rounding,
                                                            seed & (2**64 - 1), _ptr(ql), _ptr(sl), _ptr(qf),
                                                            _ptr(sf), _stream_ptr(stream)))
    return ql, sl, qf, sf


def mxfp4_quantize_2d(x, hadamard: int = HAD_NONE, rounding: int = RNE, seed: int = 0, want_last: bool = True,
                      want_first: bool = True, stream=None):
    """32 x 32 block scaling: returns (q_last, s_last, q_first, s_first); an output not wanted is None."""
    import torch
    assert x.is_cuda and x.dtype == torch.bfloat16 and x.dim() == 2 and (x.numel() == 0 or x.stride(1) == 1)
    rows, cols = x.shape
    ld = x.stride(0) if rows > 1 else max(cols, x.stride(0))
    u8 = dict(dtype=torch.uint8, device=x.device)
    ql = sl = qf = sf = None
    if want_last:
        ql, sl = torch.empty((rows, cols // 2), **u8), torch.empty((rows, cols // 32), **u8)
    if want_first:
        qf, sf = torch.empty((cols, rows // 2), **u8), torch.empty((cols, rows // 32), **u8)
    _check("mxfp4_quantize_2d", lib().mxfp4_quantize_2d(_ptr(x), rows, cols, ld, hadamard, rounding,
                                                        seed & (2**64 - 1), _ptr(ql), _ptr(sl), _ptr(qf), _ptr(sf),
                                                        _stream_ptr(stream)))
    return ql, sl, qf, sf


def mxfp4_quantize_fp8(x, axis: int = AXIS_LAST, hadamard: int = HAD_NONE, seed: int = 0, q=None, s=None,
                       stream=None):
    """MXFP8 (E4M3) quantisation of x [rows][cols]: returns (q8 [R][C], s [R][C/32])."""
    import torch
    assert x.is_cuda and x.dtype == torch.bfloat16 and x.dim() == 2 and (x.numel() == 0 or x.stride(1) == 1)
    rows, cols = x.shape
    ld = x.stride(0) if rows > 1 else max(cols, x.stride(0))
    R, C = (rows, cols) if axis == AXIS_LAST else (cols, rows)
    if q is None:
        q = torch.empty((R, C), dtype=torch.uint8, device=x.device)
    if s is None:
        s = torch.empty((R, C // 32), dtype=torch.uint8, device=x.device)
    _check("mxfp4_quantize_fp8", lib().mxfp4_quantize_fp8(_ptr(x), rows, cols, ld, axis, hadamard,
                                                          seed & (2**64 - 1), _ptr(q), _ptr(s), _stream_ptr(stream)))
    return q, s


def mxfp4_quantize_fp8_dual(x, hadamard: int = HAD_NONE, seed: int = 0, stream=None):
    """Both MXFP8 quantisations of x [rows][cols] from one pass: returns (q8_last, s_last, q8_first, s_first)."""
    import torch
    assert x.is_cuda and x.dtype == torch.bfloat16 and x.dim() == 2 and (x.numel() == 0 or x.stride(1) == 1)
    rows, cols = x.shape
    ld = x.stride(0) if rows > 1 else max(cols, x.stride(0))
    u8 = dict(dtype=torch.uint8, device=x.device)
    ql, sl = torch.empty((rows, cols), **u8), torch.empty((rows, cols // 32), **u8)
    qf, sf = torch.empty((cols, rows), **u8), torch.empty((cols, rows // 32), **u8)
    _check("mxfp4_quantize_fp8_dual", lib().mxfp4_quantize_fp8_dual(_ptr(x), rows, cols, ld, hadamard,
                                                                    seed & (2**64 - 1), _ptr(ql), _ptr(sl), _ptr(qf),
                                                                    _ptr(sf), _stream_ptr(stream)))
    return ql, sl, qf, sf


def mxfp4_gemm(a_q, a_s, b_q, b_s, out=None, out_dtype: int = OUT_FP32, accumulate: bool = False, stream=None,
               a_format: int = FMT_E2M1, b_format: int = FMT_E2M1):
    """out[i][j] (+)= sum_c A[i][c] B[j][c] on canonical quantised operands (uint8 CUDA tensors); with a format
    other than E2M1 for either operand the call goes to mxfp4_gemm_fmt."""
    import torch
    Ra, C = a_q.shape[0], a_q.shape[1] * (2 if a_format == FMT_E2M1 else 1)
    Rb = b_q.shape[0]
    assert b_q.shape[1] * (2 if b_format == FMT_E2M1 else 1) == C and a_q.is_contiguous() and b_q.is_contiguous()
    assert a_s.is_contiguous() and b_s.is_contiguous()
    if out is None:
        out = torch.empty((Ra, Rb), dtype=_out_dtype(out_dtype), device=a_q.device)
    assert out.dtype == _out_dtype(out_dtype) and (out.numel() == 0 or out.stride(1) == 1)
    ld = out.stride(0) if Ra > 1 else max(Rb, out.stride(0))
    if a_format == FMT_E2M1 and b_format == FMT_E2M1:
        _check("mxfp4_gemm", lib().mxfp4_gemm(_ptr(a_q), _ptr(a_s), _ptr(b_q), _ptr(b_s), Ra, Rb, C, _ptr(out), ld,
                                              out_dtype, int(accumulate), _stream_ptr(stream)))
    else:
        _check("mxfp4_gemm_fmt", lib().mxfp4_gemm_fmt(_ptr(a_q), _ptr(a_s), a_format, _ptr(b_q), _ptr(b_s), b_format,
                                                      Ra, Rb, C, _ptr(out), ld, out_dtype, int(accumulate),
                                                      _stream_ptr(stream)))
    return out


def mxfp4_gemm_pair(a0, b0, out0, a1, b1, out1, accumulate1: bool = False, stream=None):
    """Two independent MXFP4 GEMMs enqueued together (Dgrad and Wgrad of one layer): a0, b0, a1, b1 are
    (codes, scales) pairs of uint8 CUDA tensors, out0 / out1 preallocated bf16 or fp32 matrices."""
    import torch
    args = []
    for (aq, as_), (bq, bs), out in ((a0, b0, out0), (a1, b1, out1)):
        Ra, Rb, C = aq.shape[0], bq.shape[0], aq.shape[1] * 2
        assert bq.shape[1] * 2 == C and all(t.is_contiguous() for t in (aq, as_, bq, bs))
        assert tuple(out.shape) == (Ra, Rb) and (out.numel() == 0 or out.stride(1) == 1)
        ld = out.stride(0) if Ra > 1 else max(Rb, out.stride(0))
        args += [_ptr(aq), _ptr(as_), _ptr(bq), _ptr(bs), Ra, Rb, C, _ptr(out), ld,
                 OUT_FP32 if out.dtype == torch.float32 else OUT_BF16]
    _check("mxfp4_gemm_pair", lib().mxfp4_gemm_pair(*args, int(accumulate1), _stream_ptr(stream)))
    return out0, out1


GEMM_ANY, GEMM_TILED_256, GEMM_TILED_128, GEMM_TILED_256_TAIL_128 = 0, 1, 2, 3


def mxfp4_gemm_plan(Ra: int, Rb: int, C: int, a_format: int = FMT_E2M1, b_format: int = FMT_E2M1,
                    ld_out: Optional[int] = None, compute_units: int = 256):
    """The kernels a GEMM of this shape is cut into: list of (kind, r0, rows, c0, cols, main_tiles).  Host-only."""
    n = ctypes.c_int(0)
    parts = (ctypes.c_int64 * 24)()
    _check("mxfp4_gemm_plan", lib().mxfp4_gemm_plan(Ra, Rb, C, a_format, b_format, Rb if ld_out is None else ld_out,
                                                    compute_units, ctypes.byref(n), parts))
    return [tuple(int(parts[6 * i + k]) for k in range(6)) for i in range(n.value)]


ROUTE_NONE, ROUTE_BLOCKS, ROUTE_ANY_SHAPE, ROUTE_EDGE_64, ROUTE_EDGE_128, ROUTE_EDGE_256, ROUTE_RAGGED_TILED = range(-1, 6)
PAIR_APART, PAIR_SIDE_BY_SIDE, PAIR_NARROW_BESIDE_WIDE, PAIR_EDGE = range(4)


def mxfp4_gemm_route(Ra: int, Rb: int, C: int, a_format: int = FMT_E2M1, b_format: int = FMT_E2M1,
                     ld_out: Optional[int] = None, out_dtype: int = OUT_BF16, accumulate: bool = False,
                     compute_units: int = 256) -> int:
    """What mxfp4_gemm launches for a product of this shape (ROUTE_*).  Host-only."""
    route = ctypes.c_int(0)
    _check("mxfp4_gemm_route", lib().mxfp4_gemm_route(Ra, Rb, C, a_format, b_format, Rb if ld_out is None else ld_out,
                                                      out_dtype, int(accumulate), compute_units, ctypes.byref(route)))
    return route.value


def mxfp4_gemm_pair_route(shape0, shape1, formats=(FMT_E2M1, FMT_E2M1), out_dtypes=(OUT_BF16, OUT_FP32),
                          accumulate1: bool = False, compute_units: int = 256):
    """What mxfp4_gemm_pair, or a backward call with both gradients, launches for products of shapes (Ra, Rb, C) with
    dense outputs: (PAIR_*, first, n, cut).  Host-only."""
    route = (ctypes.c_int * 4)()
    (a0, b0, c0), (a1, b1, c1) = shape0, shape1
    _check("mxfp4_gemm_pair_route", lib().mxfp4_gemm_pair_route(
        a0, b0, c0, formats[0], b0, out_dtypes[0], a1, b1, c1, formats[1], b1, out_dtypes[1], int(accumulate1),
        compute_units, route))
    return tuple(int(v) for v in route)


def mxfp4_linear_workspace_bytes(M: int, N: int, K: int, cfg: LinearCfg, bwd: bool) -> int:
    return int(lib().mxfp4_linear_workspace_bytes(M, N, K, ctypes.byref(cfg), int(bwd)))


def _cfg_ref(cfg):
    return None if cfg is None else ctypes.byref(cfg)


def mxfp4_linear_workspace_layout(M: int, N: int, K: int, bwd: bool, cfg: Optional[LinearCfg] = None):
    arr = (ctypes.c_size_t * 8)()
    _check("mxfp4_linear_workspace_layout",
           lib().mxfp4_linear_workspace_layout(M, N, K, _cfg_ref(cfg), int(bwd), arr))
    return [int(v) for v in arr]


def make_cfg(hadamard: int = HAD_NONE, rounding: int = RNE, seed: int = 0, y_dtype: int = OUT_BF16,
             dx_dtype: int = OUT_BF16, dw_dtype: int = OUT_FP32, dw_accumulate: bool = False,
             geometry: int = GEOM_1D, fprop_format: int = FMT_E2M1, dgrad_format: int = FMT_E2M1,
             wgrad_format: int = FMT_E2M1) -> LinearCfg:
    return LinearCfg(hadamard, rounding, seed & (2**64 - 1), y_dtype, dx_dtype, dw_dtype, int(dw_accumulate),
                     geometry, fprop_format, dgrad_format, wgrad_format)


def mxfp4_linear_fwd(x, w, cfg: LinearCfg, y=None, workspace=None, stream=None):
    """Y = Q(X H) Q(W H)^T.  x [M][K], w [N][K] bf16 CUDA, contiguous.  Returns (y, workspace)."""
    import torch
    M, K = x.shape
    N = w.shape[0]
    assert w.shape[1] == K and x.is_contiguous() and w.is_contiguous()
    need = mxfp4_linear_workspace_bytes(M, N, K, cfg, False)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
    if y is None:
        y = torch.empty((M, N), dtype=_out_dtype(cfg.y_dtype), device=x.device)
    _check("mxfp4_linear_fwd", lib().mxfp4_linear_fwd(_ptr(x), _ptr(w), _ptr(y), M, N, K, ctypes.byref(cfg),
                                                      _ptr(workspace), workspace.numel(), _stream_ptr(stream)))
    return y, workspace


STATIC_SCRATCH_BYTES = 32 << 20


def mxfp4_linear_fwd_static(x, w, cfg: LinearCfg, y, stream=None):
    """mxfp4_linear_fwd on the library's own static device scratch: no workspace, nothing allocated (y is the
    caller's).  Returns y."""
    M, K = x.shape
    N = w.shape[0]
    assert w.shape[1] == K and x.is_contiguous() and w.is_contiguous() and y.is_contiguous()
    _check("mxfp4_linear_fwd_static", lib().mxfp4_linear_fwd_static(_ptr(x), _ptr(w), _ptr(y), M, N, K,
                                                                    ctypes.byref(cfg), _stream_ptr(stream)))
    return y


def mxfp4_linear_bwd(dy, x, w, cfg: LinearCfg, dx=None, dw=None, need_dx: bool = True, need_dw: bool = True,
                     workspace=None, stream=None):
    """dX = Q(dY H) Q(W^T H)^T and dW = Q(dY^T H) Q(X^T H)^T.  Returns (dx, dw, workspace)."""
    import torch
    M, N = dy.shape
    K = x.shape[1] if x is not None else w.shape[1]
    need = mxfp4_linear_workspace_bytes(M, N, K, cfg, True)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=dy.device)
    if need_dx and dx is None:
        dx = torch.empty((M, K), dtype=_out_dtype(cfg.dx_dtype), device=dy.device)
    if need_dw and dw is None:
        assert not cfg.dw_accumulate, "accumulating into dW needs the caller's dW"
        dw = torch.empty((N, K), dtype=_out_dtype(cfg.dw_dtype), device=dy.device)
    _check("mxfp4_linear_bwd", lib().mxfp4_linear_bwd(_ptr(dy), _ptr(x), _ptr(w), _ptr(dx) if need_dx else None,
                                                      _ptr(dw) if need_dw else None, M, N, K, ctypes.byref(cfg),
                                                      _ptr(workspace), workspace.numel(), _stream_ptr(stream)))
    return dx, dw, workspace


def mxfp4_linear_saved_bytes(M: int, N: int, K: int, cfg: Optional[LinearCfg] = None) -> int:
    return int(lib().mxfp4_linear_saved_bytes(M, N, K, _cfg_ref(cfg)))


def mxfp4_linear_saved_layout(M: int, N: int, K: int, cfg: Optional[LinearCfg] = None):
    arr = (ctypes.c_size_t * 4)()
    _check("mxfp4_linear_saved_layout", lib().mxfp4_linear_saved_layout(M, N, K, _cfg_ref(cfg), arr))
    return [int(v) for v in arr]


def mxfp4_linear_fwd_save(x, w, cfg: LinearCfg, y=None, workspace=None, saved=None, stream=None):
    """mxfp4_linear_fwd that also leaves the column-wise quantisations of W and X in `saved` for
    mxfp4_linear_bwd_saved.  Returns (y, workspace, saved)."""
    import torch
    M, K = x.shape
    N = w.shape[0]
    assert w.shape[1] == K and x.is_contiguous() and w.is_contiguous()
    if workspace is None:
        workspace = torch.empty(mxfp4_linear_workspace_bytes(M, N, K, cfg, False), dtype=torch.uint8, device=x.device)
    if saved is None:
        saved = torch.empty(mxfp4_linear_saved_bytes(M, N, K, cfg), dtype=torch.uint8, device=x.device)
    if y is None:
        y = torch.empty((M, N), dtype=_out_dtype(cfg.y_dtype), device=x.device)
    _check("mxfp4_linear_fwd_save", lib().mxfp4_linear_fwd_save(
        _ptr(x), _ptr(w), _ptr(y), M, N, K, ctypes.byref(cfg), _ptr(workspace), workspace.numel(), _ptr(saved),
        saved.numel(), _stream_ptr(stream)))
    return y, workspace, saved


def mxfp4_linear_bwd_saved(dy, saved, K: int, cfg: LinearCfg, dx=None, dw=None, need_dx: bool = True,
                           need_dw: bool = True, workspace=None, stream=None):
    """Dgrad and Wgrad against the operands mxfp4_linear_fwd_save left in `saved`.  Returns (dx, dw, workspace)."""
    import torch
    M, N = dy.shape
    assert dy.is_contiguous()
    if workspace is None:
        workspace = torch.empty(mxfp4_linear_workspace_bytes(M, N, K, cfg, True), dtype=torch.uint8, device=dy.device)
    if need_dx and dx is None:
        dx = torch.empty((M, K), dtype=_out_dtype(cfg.dx_dtype), device=dy.device)
    if need_dw and dw is None:
        assert not cfg.dw_accumulate, "accumulating into dW needs the caller's dW"
        dw = torch.empty((N, K), dtype=_out_dtype(cfg.dw_dtype), device=dy.device)
    _check("mxfp4_linear_bwd_saved", lib().mxfp4_linear_bwd_saved(
        _ptr(dy), _ptr(saved), saved.numel(), _ptr(dx) if need_dx else None, _ptr(dw) if need_dw else None, M, N, K,
        ctypes.byref(cfg), _ptr(workspace), workspace.numel(), _stream_ptr(stream)))
    return dx, dw, workspace


# ---- around a linear layer ------------------------------------------------------------
def make_norm_cfg(eps: float = 1e-5, residual_scale: float = 1.0, branch_scale: float = 1.0, weight_offset: float = 0.0,
                  post_norm: bool = False, accumulate: bool = False) -> NormCfg:
    return NormCfg(eps, residual_scale, branch_scale, weight_offset, int(post_norm), int(accumulate))


def _types():
    """{torch type: its code} of the types that the calls around a linear layer take."""
    global _type_codes, _fp32
    if _type_codes is None:
        import torch
        _type_codes, _fp32 = {torch.float32: OUT_FP32, torch.bfloat16: OUT_BF16}, torch.float32
    return _type_codes


_type_codes = _fp32 = None


def _empty(shape, dtype, device, stream):
    """A tensor of the call's stream: the allocator keeps what the caller drops from other streams while that one works on it."""
    import torch
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


# (On the host these calls take as long as a small one does on the GPU: what is asked of a tensor is asked once.)
def _rows_of(t, shape, dtype):
    """(pointer, leading dimension) of a CUDA matrix of this shape with unit inner stride; (None, 0) for None."""
    if t is None:
        return None, 0
    ld, inner = t.stride()
    assert t.is_cuda and t.dtype is dtype and t.shape == shape and (inner == 1 or shape[1] == 1 or not shape[0])
    return t.data_ptr(), (ld if shape[0] > 1 else max(shape[1], ld))


def _vector(t, n: int):
    """Pointer of a dense fp32 CUDA vector; None for None."""
    if t is None:
        return None
    assert t.is_cuda and t.dtype is _fp32 and t.shape == (n,) and (t.stride(0) == 1 or n == 1)
    return t.data_ptr()


def _gate(call: str, gate, shape, dtype):
    if gate is None:
        return None, 0
    if gate.dim() == 1:
        return _vector(gate, shape[1]), 0
    p, ld = _rows_of(gate, shape, dtype)
    if ld == 0:  # one row broadcast over all: refused here as the calls refuse it of any other operand, since of a gate 0 means an fp32 vector to them
        raise Mxfp4Error(call, ESHAPE)
    return p, ld


def mxfp4_residual_norm_fwd(x, o, cfg: NormCfg, gate=None, w_post=None, w_pre=None, x_out=None, h=None, rstd=None,
                            want_x_out: bool = True, want_h: bool = True, branch_dtype=None, stream=None):
    """x' = residual_scale x + branch_scale gate n(o) and h = norm(x').  x [rows][cols] bf16 or fp32; o (or None), a gate per row and
    h share a type of their own (branch_dtype where there is no o: bf16 unless given); a gate [cols] and the weights are fp32.  A gate per row has
    rows of its own (one broadcast over them is refused: it is the gate [cols], in fp32).
    Returns (x_out, h, rstd); an output not wanted is None."""
    shape, x_type, codes = x.shape, x.dtype, _types()
    rows, cols = shape
    branch = o.dtype if o is not None else h.dtype if h is not None else branch_dtype
    if x_out is None or h is None or rstd is None or branch is None:
        import torch
        branch = branch or torch.bfloat16
        if x_out is None and want_x_out:
            x_out = _empty(shape, x_type, x.device, stream)
        if h is None and want_h:
            h = _empty(shape, branch, x.device, stream)
        if rstd is None:
            rstd = _empty((2, rows), torch.float32, x.device, stream)
    assert rstd.is_cuda and rstd.dtype is _fp32 and rstd.shape == (2, rows) and rstd.is_contiguous()
    _check("mxfp4_residual_norm_fwd", lib().mxfp4_residual_norm_fwd(
        *_rows_of(x, shape, x_type), *_rows_of(o, shape, branch), *_gate("mxfp4_residual_norm_fwd", gate, shape, branch),
        _vector(w_post, cols), _vector(w_pre, cols), rows, cols, codes[x_type], codes[branch], ctypes.byref(cfg),
        *_rows_of(x_out, shape, x_type), *_rows_of(h, shape, branch), rstd.data_ptr(), _stream_ptr(stream)))
    return x_out, h, rstd


def mxfp4_residual_norm_workspace_bytes(rows: int, cols: int) -> int:
    return int(lib().mxfp4_residual_norm_workspace_bytes(rows, cols))


def mxfp4_residual_norm_bwd(dx_out, dh, x_out, o, rstd, cfg: NormCfg, gate=None, w_post=None, w_pre=None, dx=None, do=None, dgate=None,
                            dw_post=None, dw_pre=None, workspace=None, stream=None):
    """Gradients of mxfp4_residual_norm_fwd, into those of dx, do, dgate, dw_post and dw_pre that are given (dx_out or dh may be None).
    The workspace is allocated here unless passed in; returned."""
    codes = _types()
    shape = (dh if dx_out is None else dx_out).shape
    rows, cols = shape
    x_type = (dx_out if dx_out is not None else x_out).dtype
    branch = o if o is not None else dh if dh is not None else do
    branch = x_type if branch is None else branch.dtype
    if workspace is None:
        import torch
        workspace = _empty(mxfp4_residual_norm_workspace_bytes(rows, cols), torch.uint8, (dh if dx_out is None else dx_out).device, stream)
    if rstd is not None:
        assert rstd.is_cuda and rstd.dtype is _fp32 and rstd.shape == (2, rows) and rstd.is_contiguous()
    assert gate is None or dgate is None or dgate.dim() == gate.dim()
    _check("mxfp4_residual_norm_bwd", lib().mxfp4_residual_norm_bwd(
        *_rows_of(dx_out, shape, x_type), *_rows_of(dh, shape, branch), *_rows_of(x_out, shape, x_type), *_rows_of(o, shape, branch),
        *_gate("mxfp4_residual_norm_bwd", gate, shape, branch), _vector(w_post, cols), _vector(w_pre, cols), _ptr(rstd),
        rows, cols, codes[x_type], codes[branch], ctypes.byref(cfg), *_rows_of(dx, shape, x_type), *_rows_of(do, shape, branch),
        *_gate("mxfp4_residual_norm_bwd", dgate, shape, branch), _vector(dw_post, cols), _vector(dw_pre, cols), workspace.data_ptr(), workspace.numel(), _stream_ptr(stream)))
    return workspace


def make_rope_cfg(base: float = 10000.0, scaling: int = ROPE_SCALE_NONE, factor: float = 1.0, low: float = 1.0, high: float = 32.0,
                  original_positions: float = 8192.0, attention_factor: float = 0.0) -> RopeCfg:
    return RopeCfg(base, factor, low, high, original_positions, attention_factor, scaling)


def mxfp4_rope_table(positions: int, rot_dim: int, cfg: RopeCfg, table=None, device="cuda", stream=None):
    """cos and sin of positions 0 .. positions - 1: fp32 [positions][rot_dim / 2][2]."""
    import torch
    if table is None:
        table = _empty((positions, rot_dim // 2, 2), torch.float32, device, stream)
    assert table.is_cuda and table.dtype == torch.float32 and tuple(table.shape) == (positions, rot_dim // 2, 2) and table.is_contiguous()
    _check("mxfp4_rope_table", lib().mxfp4_rope_table(_ptr(table), positions, rot_dim, ctypes.byref(cfg), _stream_ptr(stream)))
    return table


def mxfp4_rope(x, table, positions=None, first_position: int = 0, rot_dim: Optional[int] = None, layout: int = ROPE_HALF,
               inverse: bool = False, out=None, stream=None):
    """Turns the first rot_dim elements (all that the table has, unless given) of the heads of x [tokens][heads][head_dim], any strides but a unit
    inner one, by their tokens' positions (int32 [tokens], or first_position + t).  out may be x; allocated here unless passed in.  inverse: the gradient, which turns the
    other way and multiplies by the table's attention factor as the forward call does."""
    shape, dtype, codes = x.shape, x.dtype, _types()
    tokens, heads, dim = shape
    known, pairs, two = table.shape
    rot = 2 * pairs if rot_dim is None else rot_dim
    if out is None:
        out = _empty(shape, dtype, x.device, stream)
    x_token, x_head, x_inner = x.stride()
    out_token, out_head, out_inner = out.stride()
    assert x.is_cuda and out.is_cuda and out.dtype == dtype and out.shape == shape and x_inner == 1 and out_inner == 1
    assert table.is_cuda and table.dtype is _fp32 and table.is_contiguous() and two == 2 and 2 * pairs == rot
    if positions is not None:
        import torch
        assert positions.is_cuda and positions.dtype == torch.int32 and positions.shape == (tokens,) and positions.is_contiguous()
    _check("mxfp4_rope", lib().mxfp4_rope(x.data_ptr(), x_token, x_head, out.data_ptr(), out_token, out_head, tokens, heads, dim, rot,
                                          codes[dtype], layout, int(inverse), _ptr(positions), first_position, table.data_ptr(), known,
                                          _stream_ptr(stream)))
    return out


def make_muon_cfg(steps: int = 5, a: float = 3.4445, b: float = -4.775, c: float = 2.0315, momentum: float = 0.95, nesterov: bool = True,
                  eps: float = 1e-7, out_scale: float = 1.0, join_steps: bool = False) -> MuonCfg:
    """join_steps: two and three steps in one where that is faster; the result is then within 5e-3 of the formula's instead of 1e-3 (root of the sum of
    squares, before its rounding to bf16)."""
    return MuonCfg(momentum, int(nesterov), steps, a, b, c, eps, out_scale, int(join_steps))


def mxfp4_orthogonalize_workspace_bytes(batch: int, N: int, K: int) -> int:
    return int(lib().mxfp4_orthogonalize_workspace_bytes(batch, N, K))


def mxfp4_orthogonalize(g, cfg: MuonCfg, momentum=None, out=None, workspace=None, stream=None):
    """The orthogonalised update (bf16) of a gradient g [N][K], or of each of g [batch][N][K], fp32 or bf16 with a unit inner stride.
    momentum (fp32, dense, of g's shape) is updated in place.  Returns (out, workspace)."""
    import torch
    batch = g.shape[0] if g.dim() == 3 else 1
    N, K = g.shape[-2:]
    if out is None:
        out = _empty(g.shape, torch.bfloat16, g.device, stream)
    assert g.is_cuda and g.dim() in (2, 3) and out.is_cuda and out.shape == g.shape and out.dtype == torch.bfloat16
    assert g.numel() == 0 or K == 1 or (g.stride(-1) == 1 and out.stride(-1) == 1)
    if momentum is not None:
        assert momentum.is_cuda and momentum.dtype == torch.float32 and momentum.shape == g.shape and momentum.is_contiguous()
    if workspace is None:
        workspace = _empty(mxfp4_orthogonalize_workspace_bytes(batch, N, K), torch.uint8, g.device, stream)

    def strides(t):
        return t.stride(-2) if N > 1 else max(K, t.stride(-2)), t.stride(0) if t.dim() == 3 and batch > 1 else 0
    _check("mxfp4_orthogonalize", lib().mxfp4_orthogonalize(_ptr(g), *strides(g), _ptr(momentum), _ptr(out), *strides(out), batch, N, K,
                                                            _types()[g.dtype], ctypes.byref(cfg), _ptr(workspace), workspace.numel(),
                                                            _stream_ptr(stream)))
    return out, workspace
