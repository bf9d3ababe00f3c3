"""Thin ctypes binding over libnvfp4.so: argument marshalling only.

Every function has the name of the C entry point it calls (include/nvfp4.h).
torch tensors are used for device memory and streams; all computation happens
inside the CUDA library.  There is no CPU fallback: if the library is missing
or a call fails, an exception is raised.

The calls that launch work go through the extension module _calls (csrc/python_calls.cpp says how it takes its
arguments), the queries through ctypes.

A call that is given a stream runs there, and what it allocates is that stream's: its scratch, and the outputs that are
not given.  They may be passed on to further calls on that stream and dropped at any time; the caller lets the streams
wait for one another as for any tensor.
"""
import ctypes as C
import functools
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libnvfp4.so")

BF16, FP32 = 0, 1
RTN, SR = 0, 1
SF_LINEAR, SF_SWIZZLED = 0, 1
G_NONE, G_AMAX, G_GIVEN = 0, 1, 2
LINEAR_FWD, LINEAR_BWD_DX, LINEAR_BWD_DW = 0, 1, 2


class NvFp4Error(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where}: nvfp4 status {status} ({status_string(status)})")


class Rounding(C.Structure):
    _fields_ = [("mode", C.c_int32), ("reserved", C.c_int32), ("seed", C.c_uint64), ("offset", C.c_uint64)]

    def __init__(self, mode=RTN, seed=0, offset=0):
        super().__init__(mode, 0, seed, offset)


_lib = None


def lib():
    """Load libnvfp4.so (built in-tree by paper_2505_19115_b200/build.py).  Raises if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} not found: build it with `python -m paper_2505_19115_b200.build` "
                           "(there is no CPU fallback)")
    L = C.CDLL(LIB_PATH)
    vp, i64, ci, sz = C.c_void_p, C.c_int64, C.c_int, C.c_size_t
    rp = C.POINTER(Rounding)
    L.nvfp4_status_string.restype = C.c_char_p
    L.nvfp4_status_string.argtypes = [ci]
    L.nvfp4_sf_bytes.restype = sz
    L.nvfp4_sf_bytes.argtypes = [i64, i64, ci]
    L.nvfp4_quantize.restype = ci
    L.nvfp4_quantize.argtypes = [vp, ci, i64, i64, i64, ci, vp, rp, vp, vp, ci, vp]
    L.nvfp4_quantize_dual.restype = ci
    L.nvfp4_quantize_dual.argtypes = [vp, ci, i64, i64, i64, vp, rp, vp, vp, rp, vp, vp, ci, vp]
    L.nvfp4_quantization_noise.restype = ci
    L.nvfp4_quantization_noise.argtypes = [vp, ci, i64, i64, i64, ci, vp, vp, vp, ci, vp, vp]
    L.nvfp4_tensor_amax_scale.restype = ci
    L.nvfp4_tensor_amax_scale.argtypes = [vp, ci, i64, i64, i64, vp, vp]
    L.nvfp4_gemm.restype = ci
    L.nvfp4_gemm.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, i64, vp, ci, i64, vp]
    L.nvfp4_gemm_quantized.restype = ci
    L.nvfp4_gemm_quantized.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, i64, vp, rp, vp, vp, ci, vp]
    L.nvfp4_gemm_set_tile_n.restype = ci
    L.nvfp4_gemm_set_tile_n.argtypes = [ci]
    L.nvfp4_linear_workspace_bytes.restype = sz
    L.nvfp4_linear_workspace_bytes.argtypes = [i64, i64, i64, ci]
    lin = [vp, vp, ci, i64, i64, i64, ci, vp, vp, rp, rp, vp, ci, vp, sz, vp]
    for name in ("nvfp4_linear_fwd", "nvfp4_linear_bwd_dx", "nvfp4_linear_bwd_dw"):
        getattr(L, name).restype = ci
        getattr(L, name).argtypes = lin
    L.nvfp4_linear_fwd_qout.restype = ci
    L.nvfp4_linear_fwd_qout.argtypes = [vp, vp, ci, i64, i64, i64, ci, vp, vp, rp, rp, vp, rp, vp, vp, ci, vp, sz, vp]
    L.nvfp4_linear_fwd_qin.restype = ci
    L.nvfp4_linear_fwd_qin.argtypes = [vp, vp, vp, vp, ci, i64, i64, i64, ci, vp, rp, vp, ci, vp, sz, vp]
    L.nvfp4_linear_saved_bytes.restype = sz
    L.nvfp4_linear_saved_bytes.argtypes = [i64, i64, i64]
    L.nvfp4_linear_fused_workspace_bytes.restype = sz
    L.nvfp4_linear_fused_workspace_bytes.argtypes = [i64, i64, i64, ci]
    L.nvfp4_linear_fwd_save.restype = ci
    L.nvfp4_linear_fwd_save.argtypes = [vp, vp, ci, i64, i64, i64, ci, vp, vp, rp, rp, rp, rp, vp, ci, vp, sz, vp, sz, vp]
    L.nvfp4_linear_bwd_saved.restype = ci
    L.nvfp4_linear_bwd_saved.argtypes = [vp, ci, i64, i64, i64, ci, vp, rp, rp, vp, sz, vp, ci, vp, ci, vp, sz, vp]
    L.nvfp4_linear_bwd.restype = ci
    L.nvfp4_linear_bwd.argtypes = [vp, vp, vp, ci, i64, i64, i64, ci, vp, vp, vp, rp, rp, rp, rp, vp, ci, vp, ci, vp, sz, vp]
    L.nvfp4_sf_bytes_mx.restype = sz
    L.nvfp4_sf_bytes_mx.argtypes = [i64, i64, ci]
    L.nvfp4_quantize_mx.restype = ci
    L.nvfp4_quantize_mx.argtypes = [vp, ci, i64, i64, i64, ci, vp, rp, vp, vp, ci, vp, sz, vp]
    L.nvfp4_gemm_mx.restype = ci
    L.nvfp4_gemm_mx.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, i64, vp, ci, i64, vp]
    L.nvfp4_gemm_bf16.restype = ci
    L.nvfp4_gemm_bf16.argtypes = [vp, vp, i64, i64, i64, vp, ci, i64, vp]
    L.nvfp4_gemm_bf16_ex.restype = ci
    L.nvfp4_gemm_bf16_ex.argtypes = [vp, ci, vp, ci, i64, i64, i64, vp, ci, i64, vp]
    L.nvfp4_transpose_bf16.restype = ci
    L.nvfp4_transpose_bf16.argtypes = [vp, i64, i64, i64, vp, vp]
    L.nvfp4_linear_bwd_bf16_workspace_bytes.restype = sz
    L.nvfp4_linear_bwd_bf16_workspace_bytes.argtypes = [i64, i64, i64]
    L.nvfp4_linear_bwd_bf16.restype = ci
    L.nvfp4_linear_bwd_bf16.argtypes = [vp, vp, vp, i64, i64, i64, vp, ci, vp, ci, vp, sz, vp]
    L.nvfp4_codes_bytes_fp8.restype = sz
    L.nvfp4_codes_bytes_fp8.argtypes = [i64, i64]
    L.nvfp4_sf_bytes_fp8.restype = sz
    L.nvfp4_sf_bytes_fp8.argtypes = [i64, i64, ci]
    L.nvfp4_linear_fp8_workspace_bytes.restype = sz
    L.nvfp4_linear_fp8_workspace_bytes.argtypes = [i64, i64, i64, ci]
    L.nvfp4_expert_rows.restype = i64
    L.nvfp4_expert_rows.argtypes = [i64, i64, i64]
    L.nvfp4_experts_fp8_workspace_bytes.restype = sz
    L.nvfp4_experts_fp8_workspace_bytes.argtypes = [i64, i64, i64, i64, i64, ci]
    L.nvfp4_quantize_fp8.restype = ci
    L.nvfp4_quantize_fp8.argtypes = [vp, ci, i64, i64, i64, i64, ci, vp, vp, vp, vp, ci, vp]
    L.nvfp4_gemm_fp8.restype = ci
    L.nvfp4_gemm_fp8.argtypes = [vp, vp, vp, vp, i64, i64, i64, vp, ci, i64, vp]
    L.nvfp4_linear_fp8_fwd.restype = ci
    L.nvfp4_linear_fp8_fwd.argtypes = [vp, vp, ci, i64, i64, i64, vp, ci, vp, sz, vp]
    L.nvfp4_linear_fp8_bwd.restype = ci
    L.nvfp4_linear_fp8_bwd.argtypes = [vp, vp, vp, ci, i64, i64, i64, vp, ci, vp, ci, vp, sz, vp]
    L.nvfp4_expert_sort.restype = ci
    L.nvfp4_expert_sort.argtypes = [vp, ci, i64, i64, i64, vp, vp, vp, vp, vp]
    L.nvfp4_expert_gather.restype = ci
    L.nvfp4_expert_gather.argtypes = [vp, ci, i64, i64, i64, i64, i64, vp, vp, vp, vp, ci, vp, vp]
    L.nvfp4_expert_combine.restype = ci
    L.nvfp4_expert_combine.argtypes = [vp, ci, i64, i64, i64, i64, vp, vp, ci, vp, vp]
    L.nvfp4_expert_combine_bwd.restype = ci
    L.nvfp4_expert_combine_bwd.argtypes = [vp, ci, i64, i64, i64, i64, i64, vp, vp, vp, vp, vp, ci, vp, vp, vp]
    L.nvfp4_quantize_fp8_experts.restype = ci
    L.nvfp4_quantize_fp8_experts.argtypes = [vp, ci, ci, i64, i64, i64, i64, i64, vp, vp, vp, ci, vp, vp, vp, vp, vp]
    L.nvfp4_gemm_fp8_experts.restype = ci
    L.nvfp4_gemm_fp8_experts.argtypes = [vp, vp, vp, vp, i64, i64, i64, vp, vp, i64, i64, vp, ci, i64, vp]
    L.nvfp4_gemm_fp8_experts_dw.restype = ci
    L.nvfp4_gemm_fp8_experts_dw.argtypes = [vp, vp, vp, vp, i64, i64, i64, vp, i64, i64, vp, ci, vp]
    L.nvfp4_experts_fp8_fwd.restype = ci
    L.nvfp4_experts_fp8_fwd.argtypes = [vp, ci, vp, ci, i64, i64, i64, i64, i64, vp, vp, vp, ci, vp, sz, vp]
    L.nvfp4_experts_fp8_bwd.restype = ci
    L.nvfp4_experts_fp8_bwd.argtypes = [vp, ci, vp, ci, vp, vp, ci, ci, i64, i64, i64, i64, i64, vp, vp, vp, ci, vp, ci, vp, sz, vp]
    L.nvfp4_linear_fwd_static.restype = ci
    L.nvfp4_linear_fwd_static.argtypes = [vp, vp, ci, i64, i64, i64, ci, vp, vp, rp, rp, vp, ci, vp]
    L.nvfp4_microbench_mma_peak.restype = ci
    L.nvfp4_microbench_mma_peak.argtypes = [ci, ci, vp, sz, C.POINTER(C.c_int), vp]
    L.nvfp4_device_error_word.restype = ci
    L.nvfp4_device_error_word.argtypes = [C.POINTER(C.c_uint32)]
    _lib = L
    return L


_calls = None


def _native():
    """The extension module, bound to the library that lib() loaded."""
    global _calls
    if _calls is None:
        lib()
        try:
            from . import _calls as module
        except ImportError as e:
            raise RuntimeError(f"the extension module _calls cannot be imported ({e}): build it with "
                               "`python -m paper_2505_19115_b200.build`") from e
        module.bind(LIB_PATH, Rounding)
        _calls = module
    return _calls


def status_string(status: int) -> str:
    return lib().nvfp4_status_string(status).decode()


def _check(status, where):
    if status != 0:
        raise NvFp4Error(status, where)


_DTYPE_CODES = {torch.bfloat16: BF16, torch.float32: FP32}


def _dtype_code(t: torch.Tensor) -> int:
    code = _DTYPE_CODES.get(t.dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {t.dtype}")
    return code


def _ptr(t):
    return None if t is None else t.data_ptr()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)     # not part of torch's public interface


def _stream(stream=None):
    """Handle of `stream`, or of the current stream of the current device.  The small calls are bound by the host, so
    the handle is fetched without building a torch.cuda.Stream object (1.3 us of a call)."""
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _empty(size, dtype, like, stream):
    """An output of a call on `stream` (None: the current stream), on the device of the tensor `like`."""
    if stream is None:
        return torch.empty(size, dtype=dtype, device=like.device)
    return _native().empty_on(stream, like, dtype or torch.get_default_dtype(), 1, *size)


def _scratch(nbytes, like, given, stream):
    """The workspace of a call on `stream`: `given`, or one that nothing else uses before the call's kernels are done with it."""
    if given is not None:
        return given
    if stream is None:
        return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=like.device)
    return _native().empty_on(stream, like, torch.uint8, 0, max(nbytes, 256))


def nvfp4_sf_bytes(Rq: int, Kq: int, sf_layout: int = SF_SWIZZLED) -> int:
    return int(lib().nvfp4_sf_bytes(Rq, Kq, sf_layout))


def nvfp4_quantize(x: torch.Tensor, transposed: bool = False, global_scale: torch.Tensor = None,
                   rounding: Rounding = None, sf_layout: int = SF_LINEAR, codes: torch.Tensor = None,
                   scales: torch.Tensor = None, stream=None):
    """Returns (codes [Rq, Kq/2] u8, scales u8: [Rq, Kq/16] linear or a flat swizzled buffer)."""
    assert x.is_cuda and x.dim() == 2 and x.stride(1) == 1
    rows, cols = x.shape
    Rq, Kq = (cols, rows) if transposed else (rows, cols)
    rounding = rounding or Rounding()
    if codes is None:
        codes = _empty((Rq, max(Kq // 2, 1)), torch.uint8, x, stream)
    if scales is None:
        if sf_layout == SF_LINEAR:
            scales = _empty((Rq, max(Kq // 16, 1)), torch.uint8, x, stream)
        else:
            scales = _empty((max(nvfp4_sf_bytes(Rq, Kq, sf_layout), 16),), torch.uint8, x, stream)
    st = _native().nvfp4_quantize(x, x, rows, cols, x.stride(0), int(transposed), global_scale, rounding, codes, scales,
                                  sf_layout, stream)
    _check(st, "nvfp4_quantize")
    return codes, scales


def nvfp4_quantize_dual(x: torch.Tensor, global_scale: torch.Tensor = None, rounding_row: Rounding = None,
                        rounding_t: Rounding = None, sf_layout: int = SF_LINEAR, stream=None):
    """Row and transposed quantization from one read.  Returns (codes_row, scales_row, codes_t, scales_t)."""
    assert x.is_cuda and x.dim() == 2 and x.stride(1) == 1
    rows, cols = x.shape
    rounding_row = rounding_row or Rounding()
    rounding_t = rounding_t or Rounding()

    def bufs(Rq, Kq):
        codes = _empty((Rq, max(Kq // 2, 1)), torch.uint8, x, stream)
        if sf_layout == SF_LINEAR:
            return codes, _empty((Rq, max(Kq // 16, 1)), torch.uint8, x, stream)
        return codes, _empty((max(nvfp4_sf_bytes(Rq, Kq, sf_layout), 16),), torch.uint8, x, stream)

    cr, sr = bufs(rows, cols)
    ct, stt = bufs(cols, rows)
    st = _native().nvfp4_quantize_dual(x, x, rows, cols, x.stride(0), global_scale, rounding_row, cr, sr, rounding_t,
                                       ct, stt, sf_layout, stream)
    _check(st, "nvfp4_quantize_dual")
    return cr, sr, ct, stt


def nvfp4_quantization_noise(x: torch.Tensor, codes, scales, transposed: bool = False, global_scale=None,
                             sf_layout: int = SF_LINEAR, stream=None) -> torch.Tensor:
    """Device tensor of two doubles: sum (Q(x) - x)^2 and sum x^2 (Section 4's noise and norm)."""
    assert x.is_cuda and x.dim() == 2 and x.stride(1) == 1
    sums = _empty((2,), torch.float64, x, stream)
    st = lib().nvfp4_quantization_noise(_ptr(x), _dtype_code(x), x.shape[0], x.shape[1], x.stride(0), int(transposed),
                                        _ptr(global_scale), _ptr(codes), _ptr(scales), sf_layout, _ptr(sums),
                                        _stream(stream))
    _check(st, "nvfp4_quantization_noise")
    return sums


def nvfp4_tensor_amax_scale(x: torch.Tensor, out: torch.Tensor = None, stream=None) -> torch.Tensor:
    assert x.is_cuda and x.dim() == 2 and x.stride(1) == 1
    if out is None:
        out = _empty((1,), torch.float32, x, stream)
    st = _native().nvfp4_tensor_amax_scale(x, x, x.shape[0], x.shape[1], x.stride(0), out, stream)
    _check(st, "nvfp4_tensor_amax_scale")
    return out


def nvfp4_gemm(a_codes, a_sf, a_g, b_codes, b_sf, b_g, out_dtype=torch.float32, out: torch.Tensor = None,
               stream=None) -> torch.Tensor:
    """D[M,N] = A[M,K] . B[N,K]^T on packed codes with swizzled scales."""
    M, K = a_codes.shape[0], a_codes.shape[1] * 2
    N = b_codes.shape[0]
    if out is None:
        out = _empty((M, N), out_dtype, a_codes, stream)
    st = _native().nvfp4_gemm(a_codes, a_sf, a_g, b_codes, b_sf, b_g, M, N, K, out, out, out.stride(0), stream)
    _check(st, "nvfp4_gemm")
    return out


def nvfp4_gemm_quantized(a_codes, a_sf, a_g, b_codes, b_sf, b_g, out_global_scale=None, rounding: Rounding = None,
                         sf_layout: int = SF_LINEAR, stream=None):
    """Q(A . B^T) with blocks along N, straight from the GEMM epilogue.  Returns (codes [M, N/2], scales)."""
    M, K = a_codes.shape[0], a_codes.shape[1] * 2
    N = b_codes.shape[0]
    rounding = rounding or Rounding()
    codes = _empty((M, N // 2), torch.uint8, a_codes, stream)
    if sf_layout == SF_LINEAR:
        scales = _empty((M, N // 16), torch.uint8, a_codes, stream)
    else:
        scales = _empty((max(nvfp4_sf_bytes(M, N, sf_layout), 16),), torch.uint8, a_codes, stream)
    st = _native().nvfp4_gemm_quantized(a_codes, a_sf, a_g, b_codes, b_sf, b_g, M, N, K, out_global_scale, rounding,
                                        codes, scales, sf_layout, stream)
    _check(st, "nvfp4_gemm_quantized")
    return codes, scales


def nvfp4_gemm_set_tile_n(bn: int) -> None:
    _check(lib().nvfp4_gemm_set_tile_n(bn), "nvfp4_gemm_set_tile_n")


def nvfp4_linear_workspace_bytes(M: int, N: int, K: int, which: int) -> int:
    return int(lib().nvfp4_linear_workspace_bytes(M, N, K, which))


def _linear(name, which, a, b, M, N, K, out_shape, gscale_mode, ga, gb, ra, rb, out, out_dtype, workspace, stream):
    if out is None:
        out = _empty(out_shape, out_dtype, a, stream)
    if workspace is None:
        workspace = _scratch(nvfp4_linear_workspace_bytes(M, N, K, which), a, None, stream)
    assert a.is_contiguous() and b.is_contiguous() and out.is_contiguous() and a.dtype == b.dtype
    st = getattr(_native(), name)(a, b, a, M, N, K, gscale_mode, ga, gb, ra, rb, out, out, workspace, workspace, stream)
    _check(st, name)
    return out


def nvfp4_linear_fwd(X, W, gscale_mode=G_AMAX, gx=None, gw=None, rx=None, rw=None, out=None,
                     out_dtype=torch.float32, workspace=None, stream=None):
    """Y[M,N] = Q(X) . Q(W)^T (Eq. 1/4).  Default rounding: RtN for both."""
    (M, K), N = X.shape, W.shape[0]
    return _linear("nvfp4_linear_fwd", LINEAR_FWD, X, W, M, N, K, (M, N), gscale_mode, gx, gw,
                   rx or Rounding(RTN), rw or Rounding(RTN), out, out_dtype, workspace, stream)


def nvfp4_linear_bwd_dx(dY, W, gscale_mode=G_AMAX, gdy=None, gw=None, rdy=None, rw=None, out=None,
                        out_dtype=torch.float32, workspace=None, stream=None):
    """dX[M,K] = Q(dY) . Q(W^T)^T (Eq. 2/5).  Default rounding: SR for dY, RtN for W^T."""
    (M, N), K = dY.shape, W.shape[1]
    return _linear("nvfp4_linear_bwd_dx", LINEAR_BWD_DX, dY, W, M, N, K, (M, K), gscale_mode, gdy, gw,
                   rdy or Rounding(SR, 0, 0), rw or Rounding(RTN), out, out_dtype, workspace, stream)


def nvfp4_linear_bwd_dw(dY, X, gscale_mode=G_AMAX, gdy=None, gx=None, rdy=None, rx=None, out=None,
                        out_dtype=torch.float32, workspace=None, stream=None):
    """dW[N,K] = Q(dY^T) . Q(X^T)^T (Eq. 3/6).  Default rounding: SR for both."""
    (M, N), K = dY.shape, X.shape[1]
    return _linear("nvfp4_linear_bwd_dw", LINEAR_BWD_DW, dY, X, M, N, K, (N, K), gscale_mode, gdy, gx,
                   rdy or Rounding(SR, 0, 1), rx or Rounding(SR, 0, 2), out, out_dtype, workspace, stream)


def nvfp4_linear_fwd_qout(X, W, gy=None, ry=None, gscale_mode=G_AMAX, gx=None, gw=None, rx=None, rw=None,
                          sf_layout=SF_SWIZZLED, codes=None, scales=None, workspace=None, stream=None):
    """Forward layer whose output leaves the GEMM already quantized along N: returns (codes [M, N/2], scales)."""
    (M, K), N = X.shape, W.shape[0]
    if codes is None:
        codes = _empty((M, N // 2), torch.uint8, X, stream)
    if scales is None:
        if sf_layout == SF_LINEAR:
            scales = _empty((M, N // 16), torch.uint8, X, stream)
        else:
            scales = _empty((max(nvfp4_sf_bytes(M, N, sf_layout), 16),), torch.uint8, X, stream)
    if workspace is None:
        workspace = _scratch(nvfp4_linear_workspace_bytes(M, N, K, LINEAR_FWD), X, None, stream)
    assert X.is_contiguous() and W.is_contiguous() and X.dtype == W.dtype
    st = _native().nvfp4_linear_fwd_qout(X, W, X, M, N, K, gscale_mode, gx, gw, rx or Rounding(RTN),
                                         rw or Rounding(RTN), gy, ry or Rounding(RTN), codes, scales, sf_layout,
                                         workspace, workspace, stream)
    _check(st, "nvfp4_linear_fwd_qout")
    return codes, scales


def nvfp4_linear_fwd_qin(x_codes, x_scales, gx, W, gscale_mode=G_AMAX, gw=None, rw=None, out=None,
                         out_dtype=torch.float32, workspace=None, stream=None):
    """Forward layer for an input already quantized along K (codes [M, K/2], swizzled scales, per-tensor scale gx)."""
    M, K = x_codes.shape[0], x_codes.shape[1] * 2
    N = W.shape[0]
    if out is None:
        out = _empty((M, N), out_dtype, W, stream)
    if workspace is None:
        workspace = _scratch(nvfp4_linear_workspace_bytes(M, N, K, LINEAR_FWD), W, None, stream)
    assert W.is_contiguous() and out.is_contiguous()
    st = _native().nvfp4_linear_fwd_qin(x_codes, x_scales, gx, W, W, M, N, K, gscale_mode, gw, rw or Rounding(RTN), out,
                                        out, workspace, workspace, stream)
    _check(st, "nvfp4_linear_fwd_qin")
    return out


FUSED_FWD_SAVE, FUSED_BWD_SAVED, FUSED_BWD = 0, 1, 2


def nvfp4_linear_saved_bytes(M, N, K) -> int:
    return int(lib().nvfp4_linear_saved_bytes(M, N, K))


def nvfp4_linear_fused_workspace_bytes(M, N, K, which) -> int:
    return int(lib().nvfp4_linear_fused_workspace_bytes(M, N, K, which))


def nvfp4_linear_fwd_save(X, W, gscale_mode=G_AMAX, gx=None, gw=None, rx=None, rw=None, rxt=None, rwt=None, out=None,
                          out_dtype=torch.float32, saved=None, workspace=None, stream=None):
    """Y = Q(X) . Q(W)^T and, from the same reads, Q(X^T) and Q(W^T) into `saved` for the backward
    and update passes.  Returns (Y, saved).  Default rounding: the paper's (RtN, RtN, SR for X^T, RtN for W^T)."""
    (M, K), N = X.shape, W.shape[0]
    if out is None:
        out = _empty((M, N), out_dtype, X, stream)
    if saved is None:
        saved = _empty((max(nvfp4_linear_saved_bytes(M, N, K), 256),), torch.uint8, X, stream)
    ws = _scratch(nvfp4_linear_fused_workspace_bytes(M, N, K, FUSED_FWD_SAVE), X, workspace, stream)
    st = _native().nvfp4_linear_fwd_save(X, W, X, M, N, K, gscale_mode, gx, gw, rx or Rounding(RTN),
                                         rw or Rounding(RTN), rxt or Rounding(SR, 0, 2), rwt or Rounding(RTN), out, out,
                                         saved, saved, ws, ws, stream)
    _check(st, "nvfp4_linear_fwd_save")
    return out, saved


def nvfp4_linear_bwd_saved(dY, saved, K, gscale_mode=G_AMAX, gdy=None, rdy=None, rdyt=None, dX=None, dW=None,
                           dx_dtype=torch.float32, dw_dtype=torch.float32, workspace=None, stream=None):
    """dX and dW from one read of dY and the operands nvfp4_linear_fwd_save kept.  Returns (dX, dW)."""
    M, N = dY.shape
    if dX is None:
        dX = _empty((M, K), dx_dtype, dY, stream)
    if dW is None:
        dW = _empty((N, K), dw_dtype, dY, stream)
    ws = _scratch(nvfp4_linear_fused_workspace_bytes(M, N, K, FUSED_BWD_SAVED), dY, workspace, stream)
    st = _native().nvfp4_linear_bwd_saved(dY, dY, M, N, K, gscale_mode, gdy, rdy or Rounding(SR, 0, 0),
                                          rdyt or Rounding(SR, 0, 1), saved, saved, dX, dX, dW, dW, ws, ws, stream)
    _check(st, "nvfp4_linear_bwd_saved")
    return dX, dW


def nvfp4_linear_bwd(dY, W, X, gscale_mode=G_AMAX, gdy=None, gw=None, gx=None, rdy=None, rdyt=None, rwt=None, rxt=None,
                     dX=None, dW=None, dx_dtype=torch.float32, dw_dtype=torch.float32, workspace=None, stream=None):
    """dX and dW (Eq. 2/5 and Eq. 3/6) with dY read once.  Returns (dX, dW)."""
    (M, N), K = dY.shape, W.shape[1]
    if dX is None:
        dX = _empty((M, K), dx_dtype, dY, stream)
    if dW is None:
        dW = _empty((N, K), dw_dtype, dY, stream)
    ws = _scratch(nvfp4_linear_fused_workspace_bytes(M, N, K, FUSED_BWD), dY, workspace, stream)
    st = _native().nvfp4_linear_bwd(dY, W, X, dY, M, N, K, gscale_mode, gdy, gw, gx, rdy or Rounding(SR, 0, 0),
                                    rdyt or Rounding(SR, 0, 1), rwt or Rounding(RTN), rxt or Rounding(SR, 0, 2), dX, dX,
                                    dW, dW, ws, ws, stream)
    _check(st, "nvfp4_linear_bwd")
    return dX, dW


def nvfp4_sf_bytes_mx(Rq: int, Kq: int, sf_layout: int = SF_SWIZZLED) -> int:
    return int(lib().nvfp4_sf_bytes_mx(Rq, Kq, sf_layout))


def nvfp4_quantize_mx(x, transposed: bool = False, global_scale=None, rounding: Rounding = None,
                      sf_layout: int = SF_LINEAR, stream=None):
    """MXFP4 (blocks of 32, E8M0 scales).  Returns (codes [Rq, Kq/2], scales: [Rq, Kq/32] or a flat swizzled buffer)."""
    assert x.is_cuda and x.dim() == 2 and x.stride(1) == 1
    rows, cols = x.shape
    Rq, Kq = (cols, rows) if transposed else (rows, cols)
    rounding = rounding or Rounding()
    codes = _empty((Rq, Kq // 2), torch.uint8, x, stream)
    if sf_layout == SF_LINEAR:
        scales = _empty((Rq, Kq // 32), torch.uint8, x, stream)
    else:
        scales = _empty((max(nvfp4_sf_bytes_mx(Rq, Kq, sf_layout), 16),), torch.uint8, x, stream)
    def call(ws):
        return _native().nvfp4_quantize_mx(x, x, rows, cols, x.stride(0), int(transposed), global_scale, rounding,
                                           codes, scales, sf_layout, ws, ws.numel() if ws is not None else 0, stream)
    st = call(None)
    if st == 5 and transposed:          # a shape the tile kernel does not take: the library transposes into a workspace first
        st = call(_scratch(rows * cols * 2, x, None, stream))
    _check(st, "nvfp4_quantize_mx")
    return codes, scales


def nvfp4_gemm_mx(a_codes, a_sf, a_g, b_codes, b_sf, b_g, out_dtype=torch.float32, out=None, stream=None):
    """D[M,N] = A[M,K] . B[N,K]^T on MXFP4 operands with swizzled E8M0 scales."""
    M, K = a_codes.shape[0], a_codes.shape[1] * 2
    N = b_codes.shape[0]
    if out is None:
        out = _empty((M, N), out_dtype, a_codes, stream)
    st = _native().nvfp4_gemm_mx(a_codes, a_sf, a_g, b_codes, b_sf, b_g, M, N, K, out, out, out.stride(0), stream)
    _check(st, "nvfp4_gemm_mx")
    return out


def nvfp4_gemm_bf16(A, B, out_dtype=torch.float32, out=None, stream=None):
    """D[M,N] = A[M,K] . B[N,K]^T on bf16 operands (the QAF phase's backward / update precision)."""
    assert A.dtype == torch.bfloat16 and B.dtype == torch.bfloat16 and A.is_contiguous() and B.is_contiguous()
    (M, K), N = A.shape, B.shape[0]
    if out is None:
        out = _empty((M, N), out_dtype, A, stream)
    _check(_native().nvfp4_gemm_bf16(A, B, M, N, K, out, out, out.stride(0), stream), "nvfp4_gemm_bf16")
    return out


def nvfp4_gemm_bf16_ex(A, a_mn_major, B, b_mn_major, out_dtype=torch.float32, out=None, stream=None):
    """D[M,N] = A . B^T on bf16 operands; an MN-major operand is passed as its stored [K, M] (or [K, N]) array."""
    assert A.dtype == torch.bfloat16 and B.dtype == torch.bfloat16 and A.is_contiguous() and B.is_contiguous()
    (K, M) = A.shape if a_mn_major else A.shape[::-1]
    N = B.shape[1] if b_mn_major else B.shape[0]
    if out is None:
        out = _empty((M, N), out_dtype, A, stream)
    _check(_native().nvfp4_gemm_bf16_ex(A, int(a_mn_major), B, int(b_mn_major), M, N, K, out, out, out.stride(0),
                                        stream), "nvfp4_gemm_bf16_ex")
    return out


def nvfp4_transpose_bf16(x, stream=None):
    assert x.dtype == torch.bfloat16 and x.dim() == 2 and x.stride(1) == 1
    out = _empty((x.shape[1], x.shape[0]), torch.bfloat16, x, stream)
    _check(lib().nvfp4_transpose_bf16(_ptr(x), x.shape[0], x.shape[1], x.stride(0), _ptr(out), _stream(stream)),
           "nvfp4_transpose_bf16")
    return out


def nvfp4_linear_bwd_bf16(dY, W, X, dx_dtype=torch.float32, dw_dtype=torch.float32, workspace=None, stream=None):
    """QAF backward + update in BF16: returns (dX[M,K], dW[N,K])."""
    (M, N), K = dY.shape, W.shape[1]
    dX = _empty((M, K), dx_dtype, dY, stream)
    dW = _empty((N, K), dw_dtype, dY, stream)
    ws = _scratch(int(lib().nvfp4_linear_bwd_bf16_workspace_bytes(M, N, K)), dY, workspace, stream)
    _check(_native().nvfp4_linear_bwd_bf16(dY, W, X, M, N, K, dX, dX, dW, dW, ws, ws, stream), "nvfp4_linear_bwd_bf16")
    return dX, dW


FP8_FWD, FP8_BWD = 0, 1


def _require(ok, call):
    """Raised, not asserted: a kernel would read or write behind a tensor that is too small."""
    if not ok:
        raise ValueError(f"{call}: a tensor is not of the size, the dtype or the layout that the call takes")


def nvfp4_codes_bytes_fp8(Rq: int, Kq: int) -> int:
    return int(lib().nvfp4_codes_bytes_fp8(Rq, Kq))


def nvfp4_sf_bytes_fp8(Rq: int, Kq: int, sf_layout: int = SF_SWIZZLED) -> int:
    return int(lib().nvfp4_sf_bytes_fp8(Rq, Kq, sf_layout))


def _product_rows(M, N, dtype, like, stream):
    """[M, N] with rows of a multiple of 16 bytes."""
    whole = 16 // dtype.itemsize
    out = _empty((M, -(-N // whole) * whole), dtype, like, stream)
    return out if N % whole == 0 else out[:, :N]


def nvfp4_quantize_fp8(x, block_rows: int = 1, row: bool = True, transposed: bool = False, sf_layout: int = SF_SWIZZLED, stream=None):
    """FP8 with a power-of-two scale for each block of 128 (block_rows 128: 128 x 128, for weights).  x [rows, cols], or dense
    [batch, rows, cols].  Returns (codes [..., rows, cols], scales, codes_t [..., cols, rows], scales_t), None for what is not wanted;
    scales: linear [..., Rq, ceil(Kq/128)], or a flat swizzled buffer."""
    out = _native().quantize_fp8(x, block_rows, row, transposed, sf_layout, stream)
    if type(out) is int:
        raise NvFp4Error(out, "nvfp4_quantize_fp8")
    return out


def nvfp4_gemm_fp8(a_codes, a_sf, b_codes, b_sf, out_dtype=torch.float32, out=None, stream=None):
    """D[M,N] = A[M,K] . B[N,K]^T on FP8 codes with swizzled scales."""
    native = _native()
    (a, M, K), (b, N, Kb) = native.fp8_operand(a_codes, a_sf), native.fp8_operand(b_codes, b_sf)
    _require(K == Kb and a == b == 1, "nvfp4_gemm_fp8")
    if out is None:
        out = _product_rows(M, N, out_dtype, a_codes, stream)
    _require(out.shape == (M, N) and out.stride(1) == 1, "nvfp4_gemm_fp8")
    st = native.nvfp4_gemm_fp8(a_codes, a_sf, b_codes, b_sf, M, N, K, out, out, out.stride(0), stream)
    _check(st, "nvfp4_gemm_fp8")
    return out


def nvfp4_linear_fp8_workspace_bytes(M: int, N: int, K: int, which: int) -> int:
    return int(lib().nvfp4_linear_fp8_workspace_bytes(M, N, K, which))


def nvfp4_linear_fp8_fwd(X, W, out=None, out_dtype=torch.float32, workspace=None, stream=None):
    """Y[M,N] = Q(X) . Q(W)^T (Eq. 1) in FP8: blocks of 1 x 128 for X, 128 x 128 for W."""
    (M, K), N = X.shape, W.shape[0]
    if out is None:
        out = _empty((M, N), out_dtype, X, stream)
    native = _native()
    _require(native.dense(X, None, M, K) and native.dense(W, X, N, K) and native.dense(out, None, M, N), "nvfp4_linear_fp8_fwd")
    if workspace is None:
        workspace = _scratch(nvfp4_linear_fp8_workspace_bytes(M, N, K, FP8_FWD), X, None, stream)
    st = native.nvfp4_linear_fp8_fwd(X, W, X, M, N, K, out, out, workspace, workspace, stream)
    _check(st, "nvfp4_linear_fp8_fwd")
    return out


def nvfp4_linear_fp8_bwd(dY, W, X, dX=None, dW=None, dx_dtype=torch.float32, dw_dtype=torch.float32, workspace=None, stream=None):
    """dX[M,K] and dW[N,K] (Eq. 2-3) in FP8, every tensor read once.  Returns (dX, dW)."""
    (M, N), K = dY.shape, W.shape[1]
    if dX is None:
        dX = _empty((M, K), dx_dtype, dY, stream)
    if dW is None:
        dW = _empty((N, K), dw_dtype, dY, stream)
    native = _native()
    _require(native.dense(dY, None, M, N) and native.dense(W, dY, N, K) and native.dense(X, dY, M, K) and
             native.dense(dX, None, M, K) and native.dense(dW, None, N, K), "nvfp4_linear_fp8_bwd")
    if workspace is None:
        workspace = _scratch(nvfp4_linear_fp8_workspace_bytes(M, N, K, FP8_BWD), dY, None, stream)
    st = native.nvfp4_linear_fp8_bwd(dY, W, X, dY, M, N, K, dX, dX, dW, dW, workspace, workspace, stream)
    _check(st, "nvfp4_linear_fp8_bwd")
    return dX, dW


@functools.lru_cache(maxsize=256)
def nvfp4_expert_rows(tokens: int, topk: int, experts: int) -> int:
    return int(lib().nvfp4_expert_rows(tokens, topk, experts))


class ExpertPlan:
    """Where the rows of every expert lie (nvfp4_expert_sort): counts [experts], offsets [experts + 1], row_of [tokens, topk] and
    slot_of [rows], int32 on the device."""
    __slots__ = ("tokens", "topk", "experts", "rows", "counts", "offsets", "row_of", "slot_of")

    def __init__(self, tokens, topk, experts, like, stream=None):
        """Buffers on the device of the tensor `like`, not filled; stream: that of the call that fills them."""
        self.tokens, self.topk, self.experts = tokens, topk, experts
        self.rows = nvfp4_expert_rows(tokens, topk, experts)
        if self.rows == 0:
            raise NvFp4Error(2, "nvfp4_expert_rows")
        self.counts, self.offsets, self.row_of, self.slot_of = _native().expert_buffers(like, tokens, topk, experts, self.rows, stream)


def nvfp4_expert_sort(expert_of, experts: int, plan: ExpertPlan = None, stream=None) -> ExpertPlan:
    """Tokens sorted by expert: expert_of [tokens, topk] (int32 or int64; an index outside [0, experts) drops the slot)."""
    wide = expert_of.dtype is torch.int64
    if not wide and expert_of.dtype is not torch.int32:
        raise TypeError(f"unsupported dtype {expert_of.dtype}")
    tokens, topk = expert_of.shape
    _require(_native().dense(expert_of, None, tokens, topk), "nvfp4_expert_sort")
    if plan is None:
        plan = ExpertPlan(tokens, topk, experts, expert_of, stream)
    else:
        _require((plan.tokens, plan.topk, plan.experts) == (tokens, topk, experts), "nvfp4_expert_sort")
    st = _native().nvfp4_expert_sort(expert_of, int(wide), tokens, topk, experts, plan.counts, plan.offsets, plan.row_of, plan.slot_of, stream)
    _check(st, "nvfp4_expert_sort")
    return plan


def _weights(weights, plan, call):
    """(tensor or None, its dtype for the call)."""
    if weights is None:
        return None, BF16
    _require(_native().dense(weights, None, plan.tokens, plan.topk), call)
    return weights, weights


def nvfp4_expert_gather(x, plan, weights=None, out=None, stream=None):
    """rows[r] = (weight *) x[token of row r], zero in padding; rows that are not used are left as they are."""
    native = _native()
    cols, ld = native.matrix(x, plan.tokens)
    if out is None:
        out = native.empty_rows(x, plan.rows, cols, stream)
    else:
        _require(native.dense(out, x, plan.rows, cols), "nvfp4_expert_gather")
    w, w_dtype = _weights(weights, plan, "nvfp4_expert_gather")
    st = native.nvfp4_expert_gather(x, x, plan.tokens, plan.topk, plan.experts, cols, ld, plan.offsets, plan.slot_of, plan.row_of,
                                    w, w_dtype, out, stream)
    _check(st, "nvfp4_expert_gather")
    return out


def nvfp4_expert_combine(rows, plan, weights=None, out=None, stream=None):
    """y[t] = sum_j (weights[t,j] *) rows[row of (t,j)]; without weights the gradient of nvfp4_expert_gather."""
    native = _native()
    cols, _ = native.matrix(rows, plan.rows)
    _require(native.dense(rows, None, plan.rows, cols), "nvfp4_expert_combine")
    if out is None:
        out = native.empty_rows(rows, plan.tokens, cols, stream)
    else:
        _require(native.dense(out, rows, plan.tokens, cols), "nvfp4_expert_combine")
    w, w_dtype = _weights(weights, plan, "nvfp4_expert_combine")
    st = native.nvfp4_expert_combine(rows, rows, plan.tokens, plan.topk, plan.experts, cols, plan.row_of, w, w_dtype, out, stream)
    _check(st, "nvfp4_expert_combine")
    return out


def nvfp4_expert_combine_bwd(dy, rows, plan, weights, rows_gradient: bool = True, drows=None, dweights=None, stream=None):
    """Gradient of nvfp4_expert_combine by its rows and its weights: (drows, or None where it is not wanted; dweights)."""
    native = _native()
    cols, ld = native.matrix(dy, plan.tokens)
    _require(native.dense(rows, dy, plan.rows, cols) and native.dense(weights, None, plan.tokens, plan.topk), "nvfp4_expert_combine_bwd")
    if drows is not None:
        _require(native.dense(drows, rows, plan.rows, cols), "nvfp4_expert_combine_bwd")
    elif rows_gradient:
        drows = native.empty_rows(rows, plan.rows, cols, stream)
    if dweights is None:
        dweights = native.empty_rows(weights, plan.tokens, plan.topk, stream)
    else:
        _require(native.dense(dweights, weights, plan.tokens, plan.topk), "nvfp4_expert_combine_bwd")
    st = native.nvfp4_expert_combine_bwd(dy, dy, plan.tokens, plan.topk, plan.experts, cols, ld, plan.offsets, plan.slot_of, plan.row_of,
                                         rows, weights, weights, drows, dweights, stream)
    _check(st, "nvfp4_expert_combine_bwd")
    return drows, dweights


def nvfp4_quantize_fp8_experts(x, plan, weights=None, sorted_rows: bool = False, row: bool = True, transposed: bool = False, stream=None):
    """nvfp4_quantize_fp8 of the sorted rows, gathered on the way from x [tokens, cols] (sorted_rows: x is [rows, cols] already) and
    multiplied by weights.  Returns (codes [rows, cols], scales, codes_t [cols, rows], scales_t)."""
    native = _native()
    cols, ld = native.matrix(x, plan.rows if sorted_rows else plan.tokens)
    out = native.empty_fp8(x, 0, plan.rows, cols, int(row), int(transposed), SF_SWIZZLED, stream)
    w, w_dtype = _weights(weights, plan, "nvfp4_quantize_fp8_experts")
    st = native.nvfp4_quantize_fp8_experts(x, x, int(not sorted_rows), plan.tokens, plan.topk, plan.experts, cols, ld, plan.offsets,
                                           plan.slot_of, w, w_dtype, *out, stream)
    _check(st, "nvfp4_quantize_fp8_experts")
    return out


def nvfp4_gemm_fp8_experts(a_codes, a_sf, b_codes, b_sf, plan, out_dtype=torch.float32, out=None, stream=None):
    """D[r] = A[r] . B[e]^T for the rows r of expert e; A [rows, K], B [experts, N, K]."""
    native = _native()
    (a, R, K), (E, N, Kb) = native.fp8_operand(a_codes, a_sf), native.fp8_operand(b_codes, b_sf)
    _require(K == Kb and a == 1 and R == plan.rows and E == plan.experts, "nvfp4_gemm_fp8_experts")
    if out is None:
        out = _product_rows(R, N, out_dtype, a_codes, stream)
    _require(out.shape == (R, N) and out.stride(1) == 1, "nvfp4_gemm_fp8_experts")
    st = native.nvfp4_gemm_fp8_experts(a_codes, a_sf, b_codes, b_sf, plan.tokens, plan.topk, E, plan.counts, plan.offsets, N, K, out, out,
                                          out.stride(0), stream)
    _check(st, "nvfp4_gemm_fp8_experts")
    return out


def nvfp4_gemm_fp8_experts_dw(a_codes, a_sf, b_codes, b_sf, plan, out_dtype=torch.float32, out=None, stream=None):
    """D[e] = A[:, rows of e] . B[:, rows of e]^T; A [N, rows], B [K, rows] (transposed outputs of nvfp4_quantize_fp8_experts)."""
    native = _native()
    (a, N, R), (b, K, Rb) = native.fp8_operand(a_codes, a_sf), native.fp8_operand(b_codes, b_sf)
    _require(a == b == 1 and R == Rb == plan.rows, "nvfp4_gemm_fp8_experts_dw")
    if out is None:
        out = _empty((plan.experts, N, K), out_dtype, a_codes, stream)
    _require(out.shape == (plan.experts, N, K) and out.is_contiguous(), "nvfp4_gemm_fp8_experts_dw")
    st = native.nvfp4_gemm_fp8_experts_dw(a_codes, a_sf, b_codes, b_sf, plan.tokens, plan.topk, plan.experts, plan.offsets, N, K, out, out, stream)
    _check(st, "nvfp4_gemm_fp8_experts_dw")
    return out


def nvfp4_experts_fp8_workspace_bytes(tokens: int, topk: int, experts: int, N: int, K: int, which: int) -> int:
    return int(lib().nvfp4_experts_fp8_workspace_bytes(tokens, topk, experts, N, K, which))


def nvfp4_experts_fp8_fwd(X, W, plan, sorted_rows: bool = False, out=None, out_dtype=None, workspace=None, stream=None):
    """Y[r] = Q(X[r]) . Q(W[e])^T for the rows r of expert e, W [experts, N, K]; X [tokens, K] is gathered on the way (sorted_rows:
    X is [rows, K] already).  Y [rows, N] of X's dtype unless told otherwise."""
    native, (E, N, K) = _native(), W.shape
    if out is None:
        out = _empty((plan.rows, N), out_dtype or X.dtype, X, stream)
    _require(native.dense(X, W, plan.rows if sorted_rows else plan.tokens, K) and native.dense(W, None, plan.experts, N, K) and
             native.dense(out, None, plan.rows, N), "nvfp4_experts_fp8_fwd")
    if workspace is None:
        workspace = _scratch(nvfp4_experts_fp8_workspace_bytes(plan.tokens, plan.topk, E, N, K, FP8_FWD), X, None, stream)
    st = native.nvfp4_experts_fp8_fwd(X, int(not sorted_rows), W, X, plan.tokens, plan.topk, E, N, K, plan.offsets, plan.slot_of, out, out,
                                      workspace, workspace, stream)
    _check(st, "nvfp4_experts_fp8_fwd")
    return out


def nvfp4_experts_fp8_bwd(dY, W, X, plan, weights=None, dy_sorted_rows: bool = False, sorted_rows: bool = False, dX=None, dW=None,
                          dx_dtype=None, dw_dtype=torch.float32, workspace=None, stream=None):
    """dX [rows, K] and dW [experts, N, K].  dY [tokens, N] is gathered on the way and multiplied by weights, as the gradient of
    nvfp4_expert_combine (dy_sorted_rows: dY is [rows, N] already); X as in nvfp4_experts_fp8_fwd.  Returns (dX, dW)."""
    native, (E, N, K) = _native(), W.shape
    if dX is None:
        dX = _empty((plan.rows, K), dx_dtype or X.dtype, dY, stream)
    if dW is None:
        dW = _empty((E, N, K), dw_dtype, dY, stream)
    _require(native.dense(dY, W, plan.rows if dy_sorted_rows else plan.tokens, N) and native.dense(X, W, plan.rows if sorted_rows else plan.tokens, K) and
             native.dense(W, None, plan.experts, N, K) and native.dense(dX, None, plan.rows, K) and native.dense(dW, None, E, N, K), "nvfp4_experts_fp8_bwd")
    w, w_dtype = _weights(weights, plan, "nvfp4_experts_fp8_bwd")
    if workspace is None:
        workspace = _scratch(nvfp4_experts_fp8_workspace_bytes(plan.tokens, plan.topk, E, N, K, FP8_BWD), dY, None, stream)
    st = native.nvfp4_experts_fp8_bwd(dY, int(not dy_sorted_rows), w, w_dtype, W, X, int(not sorted_rows), dY, plan.tokens, plan.topk, E, N, K,
                                      plan.offsets, plan.slot_of, dX, dX, dW, dW, workspace, workspace, stream)
    _check(st, "nvfp4_experts_fp8_bwd")
    return dX, dW


STATIC_WORKSPACE_BYTES = 8 << 20


def nvfp4_linear_fwd_static(X, W, gscale_mode=G_AMAX, gx=None, gw=None, rx=None, rw=None, out=None,
                            out_dtype=torch.float32, stream=None):
    """nvfp4_linear_fwd for callers that cannot allocate or pass scratch memory (for instance when
    the whole device already belongs to the host framework's pool): the scratch is a fixed
    STATIC_WORKSPACE_BYTES array inside the library, shared by all calls on a device, so calls
    that may overlap on the GPU must be serialised.  Larger layers raise (status 5)."""
    (M, K), N = X.shape, W.shape[0]
    if out is None:
        out = _empty((M, N), out_dtype, X, stream)
    rx, rw = rx or Rounding(RTN), rw or Rounding(RTN)
    assert X.is_contiguous() and W.is_contiguous() and out.is_contiguous() and X.dtype == W.dtype
    st = _native().nvfp4_linear_fwd_static(X, W, X, M, N, K, gscale_mode, gx, gw, rx, rw, out, out, stream)
    _check(st, "nvfp4_linear_fwd_static")
    return out


def nvfp4_microbench_mma_peak(stages: int, instr_n: int = 256, device=None, stream=None) -> torch.Tensor:
    """Issue-rate measurement of the FP4 tensor-core instruction: returns an int64 tensor [pairs, 3] of
    (cycles, instructions, timed-out flag) per CTA pair."""
    dev = torch.device("cuda", torch.cuda.current_device()) if device is None else device
    out = torch.zeros((torch.cuda.get_device_properties(dev).multi_processor_count // 2 + 1, 3), dtype=torch.int64, device=dev)
    if stream is not None:
        torch.cuda.current_stream(dev).synchronize()      # cleared before the kernel on that stream begins
    pairs = C.c_int(0)
    _check(lib().nvfp4_microbench_mma_peak(stages, instr_n, _ptr(out), out.numel() * 8, C.byref(pairs), _stream(stream)),
           "nvfp4_microbench_mma_peak")
    return out[:pairs.value]


def nvfp4_device_error_word() -> int:
    w = C.c_uint32(0)
    _check(lib().nvfp4_device_error_word(C.byref(w)), "nvfp4_device_error_word")
    return int(w.value)
