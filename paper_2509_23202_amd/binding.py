"""Thin binding of libfp4mr.so: argument marshalling only (ctypes; the calls of every token in compiled code, csrc/calls.cpp).

PyTorch supplies device memory (``torch.empty(..., device="cuda")``) and the current HIP stream; every step of
the path runs inside the library's HIP kernels.  There is no CPU fallback: importing this module raises if the
library has not been built (``python -m paper_2509_23202_amd.build``).
"""
from __future__ import annotations

import ctypes
import functools
from pathlib import Path

import torch

_LIB_PATH = Path(__file__).resolve().parent / "libfp4mr.so"
if not _LIB_PATH.exists():
    raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2509_23202_amd.build` "
                      "(there is no fallback path)")
lib = ctypes.CDLL(str(_LIB_PATH))

MXFP4, NVFP4 = 0, 1
GROUP = {MXFP4: 32, NVFP4: 16}

LAYOUT_GEMM = 1 << 0
INPUT_F32 = 1 << 1
STATIC_TENSOR_SCALE = 1 << 2
A_LAYOUT_GEMM = 1 << 3
W_LAYOUT_GEMM = 1 << 4
OUT_F32 = 1 << 5
SCALE_MSE = 1 << 6
SCALE_ROUND43 = 1 << 7
SCALE_FIT_TENSOR = 1 << 10
SCALE_FIT_RANGE = 1 << 11
FIT_RANGE_FLOATS = 258
SILU_MUL = 1 << 12
ROUTE_SIGMOID = 1 << 13
ROUTE_RENORM = 1 << 14
ROUTE_GROUP_SUM2 = 1 << 15
SHARED_F32 = 1 << 16
A_SCALE43 = 1 << 8
W_SCALE43 = 1 << 9
OPT_GEMM_VARIANT, OPT_GEMM_GRID, OPT_SW_CODEC, OPT_FP8_VARIANT, OPT_INT8_VARIANT = 0, 1, 2, 3, 4
OP_ROTATE_QUANTIZE, OP_QUANTIZE_WEIGHTS, OP_GEMM, OP_GPTQ, OP_GPTQ_PREPARE, OP_GPTQ_HESSIAN, OP_GEMM_SPLIT_K, OP_GEMM_FASTEST = 0, 1, 2, 3, 4, 5, 6, 7

_p, _i64, _i32, _u32, _sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_uint32, ctypes.c_size_t
_quant_sig = [_p, _i64, _i64, _i32, _i32, _p, _p, _p, _p, _sz, _u32, _p]
lib.fp4_rotate_quantize.argtypes = _quant_sig
lib.fp4_rotate_quantize.restype = _i32
lib.fp4_quantize_weights.argtypes = _quant_sig
lib.fp4_quantize_weights.restype = _i32
lib.fp4_rotate_quantize_static.argtypes = [_p, _i64, _i64, _i32, _i32, _p, _p, _p, _u32, _p]
lib.fp4_rotate_quantize_static.restype = _i32
lib.fp4_rotate_quantize_dense.argtypes = [_p, _i64, _i64, _i32, _p, _i32, _p, _p, _p, _p, _sz, _u32, _p]
lib.fp4_rotate_quantize_dense.restype = _i32
lib.fp4_fused_linear.argtypes = [_p, _i64, _i64, _i32, _p, _p, _i64, _i32, _p, _u32, _p]
lib.fp4_fused_linear.restype = _i32
lib.fp4_w4a16_linear.argtypes = lib.fp4_fused_linear.argtypes
lib.fp4_w4a16_linear.restype = _i32
lib.fp4_gptq_quantize_weights.argtypes = [_p, _i64, _i64, _i32, _i32, _p, _p, _p, _p, _p, _p, _sz, _u32, _p]
lib.fp4_gptq_quantize_weights.restype = _i32
lib.fp4_gptq_accumulate_hessian.argtypes = [_p, _i64, _i64, _i32, _p, _i32, _p, _sz, _p]
lib.fp4_gptq_accumulate_hessian.restype = _i32
lib.fp4_gptq_prepare.argtypes = [_p, _i64, ctypes.c_float, _i32, _p, _p, _p, _sz, _p]
lib.fp4_gptq_prepare.restype = _i32
lib.fp4_gemm.argtypes = [_p, _p, _p, _p, _p, _p, _i64, _i64, _i64, _i32, _p, _p, _sz, _u32, _p]
lib.fp4_gemm.restype = _i32
lib.fp4_workspace_bytes.argtypes = [_i32, _i64, _i64, _i64, _i32, _u32]
lib.fp4_workspace_bytes.restype = _sz
lib.fp4_packed_bytes.argtypes = [_i64, _i64, _i32, _u32, ctypes.POINTER(_sz), ctypes.POINTER(_sz)]
lib.fp4_packed_bytes.restype = _i32
lib.fp4_status_string.argtypes = [_i32]
lib.fp4_status_string.restype = ctypes.c_char_p
lib.fp4_version.restype = _i32
lib.fp4_probe.argtypes = [_i32, _p, _sz, _i32, _p]
lib.fp4_probe.restype = _i32
lib.fp4_dequantize.argtypes = [_p, _p, _p, _i64, _i64, _i32, _p, _u32, _p]
lib.fp4_dequantize.restype = _i32
lib.fp8_rmsnorm_quantize.argtypes = [_p, _i64, _p, _p, _i64, _i64, ctypes.c_float, _p, _p, _p, _p, _u32, _p]
lib.fp8_rmsnorm_quantize.restype = _i32
lib.fp8_quantize.argtypes = [_p, _i64, _i64, _i64, _p, _p, _u32, _p]
lib.fp8_quantize.restype = _i32
lib.fp8_quantize_weights.argtypes = [_p, _i64, _i64, _i64, _p, _p, _u32, _p]
lib.fp8_quantize_weights.restype = _i32
lib.fp8_gemm.argtypes = [_p, _p, _p, _p, _i64, _i64, _i64, _p, _p, _sz, _u32, _p]
lib.fp8_workspace_bytes.argtypes = [_i64, _i64, _i64, _u32]
lib.fp8_workspace_bytes.restype = _sz
lib.fp8_gemm.restype = _i32
lib.fp8_grouped_gemm.argtypes = [_p, _p, _i64, _p, _p, _p, _p, _i64, _i64, _i64, _i64, _p, _u32, _p]
lib.fp8_grouped_gemm.restype = _i32
lib.int8_rmsnorm_quantize.argtypes = lib.fp8_rmsnorm_quantize.argtypes
lib.int8_rmsnorm_quantize.restype = _i32
lib.int8_quantize.argtypes = lib.fp8_quantize.argtypes
lib.int8_quantize.restype = _i32
lib.int8_gemm.argtypes = lib.fp8_gemm.argtypes
lib.int8_gemm.restype = _i32
lib.int8_workspace_bytes.argtypes = [_i64, _i64, _i64]
lib.int8_workspace_bytes.restype = _sz
lib.int8_grouped_gemm.argtypes = lib.fp8_grouped_gemm.argtypes
lib.int8_grouped_gemm.restype = _i32
lib.moe_route.argtypes = [_p, _i64, _p, _i64, _i64, _i64, _i64, _i64, ctypes.c_float, _p, _p, _p, _p, _p, _p, _sz, _u32, _p]
lib.moe_route.restype = _i32
lib.moe_workspace_bytes.argtypes = [_i64, _i64, _i64]
lib.moe_workspace_bytes.restype = _sz
lib.moe_combine.argtypes = [_p, _i64, _p, _p, _p, _i64, _i64, _i64, _p, _u32, _p]
lib.moe_combine.restype = _i32
lib.fp4_set_option.argtypes = [_i32, _i32]
lib.fp4_set_option.restype = _i32


class Fp4mrError(RuntimeError):
    def __init__(self, status: int):
        self.status = status
        super().__init__(f"fp4mr status {status}: {lib.fp4_status_string(status).decode()}")


# The compiled form of the plain calls.  It answers None to everything else, and the Python below takes the call; without it (a
# torch that it was not built against) Python takes them all.
try:
    from . import _calls
    _calls.bind(*(ctypes.cast(f, _p).value for f in (lib.fp4_rotate_quantize, lib.fp4_quantize_weights, lib.fp4_rotate_quantize_dense, lib.fp4_gemm,
                                                     lib.fp4_fused_linear, lib.fp4_w4a16_linear, lib.fp4_workspace_bytes, lib.fp4_packed_bytes)), Fp4mrError)
    _calls.bind8(*(ctypes.cast(f, _p).value for f in (lib.fp8_rmsnorm_quantize, lib.fp8_quantize, lib.fp8_quantize_weights, lib.fp8_gemm, lib.fp8_workspace_bytes,
                                                       lib.fp8_grouped_gemm)))
    _calls.bind8i(*(ctypes.cast(f, _p).value for f in (lib.int8_rmsnorm_quantize, lib.int8_quantize, lib.int8_gemm, lib.int8_workspace_bytes, lib.int8_grouped_gemm, lib.moe_route,
                                                        lib.moe_workspace_bytes, lib.moe_combine)))
except ImportError:
    _calls = None


def _check(status: int) -> None:
    if status != 0:
        raise Fp4mrError(status)


# The current stream's handle without a Stream object around it: 0.2 us of host time per call, not 2.8, where a whole
# one-launch linear of a small layer takes 3 us on the GPU.
try:
    _raw_stream, _current_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
except AttributeError:   # a build of torch without these two
    _raw_stream, _current_device = (lambda device: torch.cuda.current_stream(device).cuda_stream), torch.cuda.current_device


def _stream() -> int:
    return _raw_stream(_current_device())


# Outputs come from Tensor.new_empty, which has no device argument to parse (1.3 us against torch.empty's 1.8) -- but not for a
# subclass of Tensor (a Parameter, ...), which it would hand back to the subclass: every call returns plain tensors.
_Tensor = torch.Tensor


def _plain_empty(like):
    return functools.partial(torch.empty, device=like.device)


def _ptr(t):
    return None if t is None else t.data_ptr()


@functools.lru_cache(maxsize=1024, typed=True)   # (a function of its arguments alone)
def packed_bytes(rows: int, K: int, fmt: int, flags: int = 0):
    c, s = _sz(), _sz()
    _check(lib.fp4_packed_bytes(rows, K, fmt, flags, ctypes.byref(c), ctypes.byref(s)))
    return c.value, s.value


def workspace_bytes(op: int, M: int, N: int, K: int, fmt: int, flags: int = 0) -> int:
    return int(lib.fp4_workspace_bytes(op, M, N, K, fmt, flags))


def _quantize(fn, op, x, had_block, fmt, flags, tensor_scale, codes, scales, workspace, rot=None):
    if _calls is not None and tensor_scale is None and codes is None and scales is None and workspace is None:
        out = _calls.quantize(x, had_block, fmt, flags, 2 if rot is not None else 1 if op == OP_QUANTIZE_WEIGHTS else 0, rot)
        if out is not None:
            return out
    assert x.is_cuda and x.dim() == 2 and x.is_contiguous()
    rows, K = x.shape
    if x.dtype == torch.float32:
        flags |= INPUT_F32
    elif x.dtype != torch.bfloat16:
        raise TypeError("x must be bfloat16 (or float32 with had_block=1)")
    empty = x.new_empty if type(x) is _Tensor else _plain_empty(x)
    if codes is None or scales is None:
        cb, sb = packed_bytes(rows, K, fmt, flags & LAYOUT_GEMM)
        codes = empty(cb, dtype=torch.uint8)
        scales = empty(sb, dtype=torch.uint8)
    ts = None
    if flags & SCALE_FIT_RANGE:
        # [alpha, beta, 256 scale values]; a caller-supplied tensor (its first two floats set) means: use that alpha, beta
        if tensor_scale is not None:
            assert tensor_scale.is_cuda and tensor_scale.dtype == torch.float32 and tensor_scale.numel() >= FIT_RANGE_FLOATS
            flags |= STATIC_TENSOR_SCALE
            ts = tensor_scale
        else:
            ts = torch.empty(FIT_RANGE_FLOATS, dtype=torch.float32, device=x.device)
    elif fmt == NVFP4:
        if tensor_scale is not None:
            flags |= STATIC_TENSOR_SCALE
            ts = tensor_scale
        else:
            ts = empty(1, dtype=torch.float32)
    need = workspace_bytes(op, rows, 0, K, fmt, flags)
    if need and workspace is None:
        workspace = empty(need, dtype=torch.uint8)
    wsz = 0 if workspace is None else workspace.numel()
    if rot is None:
        _check(fn(x.data_ptr(), rows, K, had_block, fmt, codes.data_ptr(), scales.data_ptr(), _ptr(ts), _ptr(workspace), wsz,
                  flags, _stream()))
    else:
        _check(fn(x.data_ptr(), rows, K, had_block, rot.data_ptr(), fmt, codes.data_ptr(), scales.data_ptr(), _ptr(ts),
                  _ptr(workspace), wsz, flags, _stream()))
    return codes, scales, ts


def fp4_rotate_quantize(x, had_block: int, fmt: int, *, flags: int = 0, tensor_scale=None, codes=None, scales=None,
                        workspace=None):
    """codes, scales, tensor_scale = Q(X H_b).  x: [M,K] bf16 cuda tensor (fp32 allowed with had_block=1).
    With flags=LAYOUT_GEMM the outputs are in the opaque GEMM layout; else canonical flat byte tensors
    (codes [M*K/2], scales [M*K/G])."""
    return _quantize(lib.fp4_rotate_quantize, OP_ROTATE_QUANTIZE, x, had_block, fmt, flags, tensor_scale, codes, scales, workspace)


def fp4_rotate_quantize_static(x, had_block: int, fmt: int, *, flags: int = 0, tensor_scale, codes, scales):
    """fp4_rotate_quantize without a workspace: the library's own static device scratch is used and nothing is allocated,
    here or in the library -- the caller passes every output (tensor_scale: a 1-element float32 cuda tensor for NVFP4,
    written unless flags has STATIC_TENSOR_SCALE; None for MXFP4)."""
    assert x.is_cuda and x.dim() == 2 and x.is_contiguous() and x.dtype == torch.bfloat16
    rows, K = x.shape
    _check(lib.fp4_rotate_quantize_static(x.data_ptr(), rows, K, had_block, fmt, codes.data_ptr(), scales.data_ptr(),
                                          _ptr(tensor_scale), flags, _stream()))
    return codes, scales, tensor_scale


def fp4_rotate_quantize_dense(x, rot, fmt: int, *, flags: int = 0, tensor_scale=None, codes=None, scales=None, workspace=None):
    """codes, scales, tensor_scale = Q(X R), R block-diagonal with the bf16 [k,k] cuda tensor `rot` on the diagonal
    (k in {16,32,64,128}); for weights pass W as x."""
    assert rot.is_cuda and rot.dtype == torch.bfloat16 and rot.dim() == 2 and rot.shape[0] == rot.shape[1] and rot.is_contiguous()
    return _quantize(lib.fp4_rotate_quantize_dense, OP_ROTATE_QUANTIZE, x, int(rot.shape[0]), fmt, flags, tensor_scale, codes,
                     scales, workspace, rot=rot)


def fp4_quantize_weights(w, had_block: int, fmt: int, *, flags: int = 0, tensor_scale=None, codes=None, scales=None,
                         workspace=None):
    """Offline RTN weight preparation, codes, scales, tensor_scale = Q(W H_b).  w: [N,K] bf16 cuda tensor."""
    return _quantize(lib.fp4_quantize_weights, OP_QUANTIZE_WEIGHTS, w, had_block, fmt, flags, tensor_scale, codes, scales, workspace)


def fp4_gptq_accumulate_hessian(x, had_block: int, hessian=None, *, workspace=None):
    """H (+)= (x H_b)^T (x H_b): x bf16 [T,K]; hessian fp32 [K,K] to add to, or None for a fresh one.  Returns hessian."""
    assert x.is_cuda and x.dim() == 2 and x.is_contiguous() and x.dtype == torch.bfloat16
    T, K = x.shape
    acc = hessian is not None
    if not acc:
        hessian = torch.empty((K, K), dtype=torch.float32, device=x.device)
    assert hessian.is_cuda and hessian.dtype == torch.float32 and hessian.is_contiguous() and tuple(hessian.shape) == (K, K)
    need = workspace_bytes(OP_GPTQ_HESSIAN, T, 0, K, MXFP4, 0)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
    _check(lib.fp4_gptq_accumulate_hessian(x.data_ptr(), T, K, had_block, hessian.data_ptr(), 1 if acc else 0,
                                           workspace.data_ptr(), workspace.numel(), _stream()))
    return hessian


def fp4_gptq_prepare(hessian, damp: float = 1e-2, act_order: bool = True, *, workspace=None):
    """Hessian fp32 [K,K] -> (perm int32 [K], hinv_u fp32 [K,K]) for fp4_gptq_quantize_weights."""
    assert hessian.is_cuda and hessian.dtype == torch.float32 and hessian.is_contiguous() and hessian.dim() == 2
    K = hessian.shape[0]
    assert hessian.shape[1] == K
    perm = torch.empty(K, dtype=torch.int32, device=hessian.device)
    U = torch.empty((K, K), dtype=torch.float32, device=hessian.device)
    need = workspace_bytes(OP_GPTQ_PREPARE, 0, 0, K, MXFP4, 0)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=hessian.device)
    _check(lib.fp4_gptq_prepare(hessian.data_ptr(), K, float(damp), 1 if act_order else 0, perm.data_ptr(), U.data_ptr(),
                                workspace.data_ptr(), workspace.numel(), _stream()))
    return perm, U


def fp4_gptq_quantize_weights(w, had_block: int, fmt: int, hinv_u, perm=None, *, flags: int = 0, workspace=None):
    """MR-GPTQ sweep: w bf16 [N,K], hinv_u fp32 [K,K] (upper factor of the damped inverse Hessian in visiting order),
    perm int32 [K] or None.  Returns (codes, scales, tensor_scale) in canonical layout."""
    assert w.is_cuda and w.dim() == 2 and w.is_contiguous() and w.dtype == torch.bfloat16
    N, K = w.shape
    assert hinv_u.is_cuda and hinv_u.dtype == torch.float32 and hinv_u.is_contiguous() and tuple(hinv_u.shape) == (K, K)
    if perm is not None:
        assert perm.is_cuda and perm.dtype == torch.int32 and perm.is_contiguous() and perm.numel() == K
    cb, sb = packed_bytes(N, K, fmt, 0)
    codes = torch.empty(cb, dtype=torch.uint8, device=w.device)
    scales = torch.empty(sb, dtype=torch.uint8, device=w.device)
    ts = torch.empty(1, dtype=torch.float32, device=w.device) if fmt == NVFP4 else None
    if flags & SCALE_FIT_RANGE:
        ts = torch.empty(FIT_RANGE_FLOATS, dtype=torch.float32, device=w.device)
    need = workspace_bytes(OP_GPTQ, N, 0, K, fmt, flags)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=w.device)
    _check(lib.fp4_gptq_quantize_weights(w.data_ptr(), N, K, had_block, fmt, hinv_u.data_ptr(), _ptr(perm), codes.data_ptr(),
                                         scales.data_ptr(), _ptr(ts), workspace.data_ptr(), workspace.numel(), flags, _stream()))
    return codes, scales, ts


def fp4_gemm(a_codes, a_scales, a_tensor_scale, w_codes, w_scales, w_tensor_scale, M: int, N: int, K: int, fmt: int, *,
             flags: int = 0, out=None, workspace=None):
    """out[M,N] = Ahat @ What^T (bf16, or fp32 with OUT_F32).  Operand layouts per A_LAYOUT_GEMM / W_LAYOUT_GEMM."""
    if _calls is not None and out is None and workspace is None:
        out = _calls.gemm(a_codes, a_scales, a_tensor_scale, w_codes, w_scales, w_tensor_scale, M, N, K, fmt, flags)
        if out is not None:
            return out
    empty = a_codes.new_empty if type(a_codes) is _Tensor else _plain_empty(a_codes)
    if out is None:
        out = empty((M, N), dtype=torch.float32 if flags & OUT_F32 else torch.bfloat16)
    need = workspace_bytes(OP_GEMM_FASTEST, M, N, K, fmt, flags)   # (what the call needs, plus split-K room where that is the faster way)
    if need and workspace is None:
        workspace = empty(need, dtype=torch.uint8)
    wsz = 0 if workspace is None else workspace.numel()
    _check(lib.fp4_gemm(a_codes.data_ptr(), a_scales.data_ptr(), _ptr(a_tensor_scale), w_codes.data_ptr(), w_scales.data_ptr(),
                        _ptr(w_tensor_scale), M, N, K, fmt, out.data_ptr(), _ptr(workspace), wsz, flags, _stream()))
    return out


def fp4_fused_linear(x, had_block: int, w_codes, w_scales, N: int, fmt: int = MXFP4, *, flags: int = 0, out=None):
    """out[M,N] = Q(X H_b) @ Q(W H_b)^T in one launch for M <= 4 tokens (MXFP4, W in GEMM layout)."""
    if _calls is not None and out is None:
        out = _calls.linear(x, had_block, w_codes, w_scales, N, fmt, flags, 0)
        if out is not None:
            return out
    assert x.is_cuda and x.dim() == 2 and x.is_contiguous() and x.dtype == torch.bfloat16
    M, K = x.shape
    if out is None:
        empty = x.new_empty if type(x) is _Tensor else _plain_empty(x)
        out = empty((M, N), dtype=torch.float32 if flags & OUT_F32 else torch.bfloat16)
    _check(lib.fp4_fused_linear(x.data_ptr(), M, K, had_block, w_codes.data_ptr(), w_scales.data_ptr(), N, fmt, out.data_ptr(),
                                flags | W_LAYOUT_GEMM, _stream()))
    return out


def fp4_w4a16_linear(x, had_block: int, w_codes, w_scales, N: int, fmt: int = MXFP4, *, flags: int = 0, out=None):
    """out[M,N] = bf16(X H_b) @ Q(W H_b)^T: weight-only variant of fp4_fused_linear (M <= 16, MXFP4, W in GEMM layout)."""
    if _calls is not None and out is None:
        out = _calls.linear(x, had_block, w_codes, w_scales, N, fmt, flags, 1)
        if out is not None:
            return out
    assert x.is_cuda and x.dim() == 2 and x.is_contiguous() and x.dtype == torch.bfloat16
    M, K = x.shape
    if out is None:
        empty = x.new_empty if type(x) is _Tensor else _plain_empty(x)
        out = empty((M, N), dtype=torch.float32 if flags & OUT_F32 else torch.bfloat16)
    _check(lib.fp4_w4a16_linear(x.data_ptr(), M, K, had_block, w_codes.data_ptr(), w_scales.data_ptr(), N, fmt, out.data_ptr(),
                                flags | W_LAYOUT_GEMM, _stream()))
    return out


PROBE_MFMA_FP4, PROBE_MFMA_F16, PROBE_COPY, PROBE_READ = 0, 1, 2, 3


def fp4_dequantize(codes, scales, tensor_scale, rows: int, K: int, fmt: int, *, flags: int = 0, out=None):
    """xhat [rows, K] = E2M1(code) * scale, bf16 (fp32 with OUT_F32), from canonical or (LAYOUT_GEMM) GEMM-layout operands.
    tensor_scale: the NVFP4 tensor scale, the FIT_RANGE_FLOATS buffer of a SCALE_FIT_RANGE call, else None."""
    assert codes.is_cuda and scales.is_cuda
    if out is None:
        out = torch.empty((rows, K), dtype=torch.float32 if flags & OUT_F32 else torch.bfloat16, device=codes.device)
    _check(lib.fp4_dequantize(codes.data_ptr(), scales.data_ptr(), _ptr(tensor_scale), rows, K, fmt, out.data_ptr(), flags, _stream()))
    return out


def fp4_probe(which: int, buf, iters: int = 1) -> None:
    """Launch one ceiling-measurement kernel on the current stream (see fp4_probe in the header); buf: cuda uint8 tensor."""
    assert buf.is_cuda and buf.is_contiguous()
    _check(lib.fp4_probe(int(which), buf.data_ptr(), buf.numel() * buf.element_size(), int(iters), _stream()))


# ---- 8-bit linear layers: E4M3 codes (torch.float8_e4m3fn) with a float32 scale per 128 columns of a row (activations: codes [M,K],
# scales [M, K/128]) or per 128 x 128 block (weights: codes [N,K], scales [ceil(N/128), K/128], or with experts in front)
FP8_BLOCK = 128
_E4M3 = torch.float8_e4m3fn


def _rows(x):
    """bf16 cuda [M, any] whose rows may be apart: (rows, elements of a row, elements between rows)."""
    assert x.is_cuda and x.dim() == 2 and x.dtype == torch.bfloat16 and (x.stride(1) == 1 or x.shape[1] <= 1)
    return x.shape[0], x.shape[1], x.stride(0) if x.shape[0] > 1 else x.shape[1]


def _fp8_outputs(x, M: int, K: int, codes, scales):
    empty = x.new_empty if type(x) is _Tensor else _plain_empty(x)
    codes = empty((M, K), dtype=_E4M3) if codes is None else codes
    scales = empty((M, K // FP8_BLOCK), dtype=torch.float32) if scales is None else scales
    _is_operand(codes, scales, (M, K), (M, K // FP8_BLOCK))
    return codes, scales


def _is_operand(codes, scales, shape, scale_shape):
    assert codes.is_cuda and codes.dtype == _E4M3 and codes.is_contiguous() and tuple(codes.shape) == shape
    assert scales.is_cuda and scales.dtype == torch.float32 and scales.is_contiguous() and tuple(scales.shape) == scale_shape


def _is_bf16(t, *shape):
    assert t.is_cuda and t.dtype == torch.bfloat16 and t.is_contiguous() and tuple(t.shape) == shape


def fp8_rmsnorm_quantize(x, weight, eps: float = 1e-6, *, residual=None, residual_out=None, norm_out=None, codes=None, scales=None):
    """codes, scales, h = Q(v) with v = h * weight / sqrt(mean(h^2) + eps) and h = bf16(x + residual), or x (then the third result is None).
    x: bf16 [M,K], rows may be apart (K % 128 == 0, K <= 65536); weight: bf16 [K]; residual: bf16 [M,K].  residual_out: where h goes (may be residual
    or x themselves, a new tensor if None); norm_out: bf16 [M,K] to receive v too."""
    if _calls is not None and residual_out is None and codes is None and scales is None:
        out = _calls.rmsnorm_quantize8(x, weight, eps, residual, norm_out)
        if out is not None:
            return out
    M, K, stride = _rows(x)
    _is_bf16(weight, K)
    empty = x.new_empty if type(x) is _Tensor else _plain_empty(x)
    if residual is not None:
        _is_bf16(residual, M, K)
        if residual_out is None:
            residual_out = empty((M, K), dtype=torch.bfloat16)
    if residual_out is not None:
        _is_bf16(residual_out, M, K)
    if norm_out is not None:
        _is_bf16(norm_out, M, K)
    codes, scales = _fp8_outputs(x, M, K, codes, scales)
    _check(lib.fp8_rmsnorm_quantize(x.data_ptr(), stride, _ptr(residual), weight.data_ptr(), M, K, eps, codes.data_ptr(), scales.data_ptr(), _ptr(residual_out),
                                    _ptr(norm_out), 0, _stream()))
    return codes, scales, residual_out


def fp8_quantize(x, *, flags: int = 0, codes=None, scales=None):
    """codes, scales = Q(x) of bf16 activations [M,K], or with SILU_MUL of silu(x[:, :K]) * x[:, K:] of x [M, 2K]; rows may be apart, K % 128 == 0."""
    if _calls is not None and codes is None and scales is None:
        out = _calls.quantize8(x, flags)
        if out is not None:
            return out
    M, K, stride = _rows(x)
    if flags & SILU_MUL:
        assert K % 2 == 0
        K //= 2
    codes, scales = _fp8_outputs(x, M, K, codes, scales)
    _check(lib.fp8_quantize(x.data_ptr(), stride, M, K, codes.data_ptr(), scales.data_ptr(), flags, _stream()))
    return codes, scales


def fp8_quantize_weights(w, *, codes=None, scales=None):
    """codes, scales = Q(w) of bf16 weights [N,K], or of experts [E,N,K]: a scale per 128 x 128 block."""
    if _calls is not None and codes is None and scales is None:
        out = _calls.quantize_weights8(w)
        if out is not None:
            return out
    assert w.is_cuda and w.dim() in (2, 3) and w.dtype == torch.bfloat16 and w.is_contiguous()
    N, K = w.shape[-2:]
    shape = (*w.shape[:-2], -(-N // FP8_BLOCK), K // FP8_BLOCK)
    empty = w.new_empty if type(w) is _Tensor else _plain_empty(w)
    codes = empty(tuple(w.shape), dtype=_E4M3) if codes is None else codes
    scales = empty(shape, dtype=torch.float32) if scales is None else scales
    _is_operand(codes, scales, tuple(w.shape), shape)
    _check(lib.fp8_quantize_weights(w.data_ptr(), w.shape[0] if w.dim() == 3 else 1, N, K, codes.data_ptr(), scales.data_ptr(), 0, _stream()))
    return codes, scales


def _product_out(a_codes, a_scales, w_codes, w_scales, dim: int, rows: int, flags: int, out):
    assert a_codes.dim() == 2 and w_codes.dim() == dim
    N, K = w_codes.shape[-2:]
    _is_operand(a_codes, a_scales, (a_codes.shape[0], K), (a_codes.shape[0], K // FP8_BLOCK))
    _is_operand(w_codes, w_scales, tuple(w_codes.shape), (*w_codes.shape[:-2], -(-N // FP8_BLOCK), K // FP8_BLOCK))
    dtype = torch.float32 if flags & OUT_F32 else torch.bfloat16
    if out is None:
        empty = a_codes.new_empty if type(a_codes) is _Tensor else _plain_empty(a_codes)
        out = empty((rows, N), dtype=dtype)
    assert out.is_cuda and out.dtype == dtype and out.is_contiguous() and tuple(out.shape) == (rows, N)
    return out, N, K


def fp8_gemm(a_codes, a_scales, w_codes, w_scales, *, flags: int = 0, out=None, workspace=None):
    """out[M,N] = A W^T (bf16, or fp32 with OUT_F32) from the codes and scales of activations [M,K] and weights [N,K]."""
    if _calls is not None and out is None and workspace is None:
        got = _calls.gemm8(a_codes, a_scales, w_codes, w_scales, flags)
        if got is not None:
            return got
    M = a_codes.shape[0]
    out, N, K = _product_out(a_codes, a_scales, w_codes, w_scales, 2, M, flags, out)
    need = fp8_workspace_bytes(M, N, K, flags)
    if need and workspace is None:
        workspace = (a_codes.new_empty if type(a_codes) is _Tensor else _plain_empty(a_codes))(need, dtype=torch.uint8)
    assert workspace is None or (workspace.is_cuda and workspace.is_contiguous())
    wsz = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib.fp8_gemm(a_codes.data_ptr(), a_scales.data_ptr(), w_codes.data_ptr(), w_scales.data_ptr(), M, N, K, out.data_ptr(), _ptr(workspace), wsz, flags, _stream()))
    return out


def fp8_workspace_bytes(M: int, N: int, K: int, flags: int = 0) -> int:
    return int(lib.fp8_workspace_bytes(M, N, K, flags))


def fp8_grouped_gemm(a_codes, a_scales, w_codes, w_scales, offsets, *, rows=None, flags: int = 0, out=None):
    """Rows offsets[e] .. offsets[e+1] - 1 of out = those rows of A times the weights of expert e, w_codes [E,N,K]; offsets: int32 cuda [E+1].
    rows: int32 cuda [T], the row of A for each row of out (outside A: a row of zeros); without it out has A's rows.  Rows of out that no expert has are
    not written (a new out holds what its memory held)."""
    if _calls is not None and out is None:
        got = _calls.gemm8(a_codes, a_scales, w_codes, w_scales, flags, offsets, rows)
        if got is not None:
            return got
    E = w_codes.shape[0]
    assert offsets.is_cuda and offsets.dtype == torch.int32 and offsets.is_contiguous() and offsets.numel() == E + 1
    T = a_codes.shape[0]
    if rows is not None:
        assert rows.is_cuda and rows.dtype == torch.int32 and rows.dim() == 1 and rows.is_contiguous()
        T = rows.shape[0]
    out, N, K = _product_out(a_codes, a_scales, w_codes, w_scales, 3, T, flags, out)
    _check(lib.fp8_grouped_gemm(a_codes.data_ptr(), a_scales.data_ptr(), a_codes.shape[0], w_codes.data_ptr(), w_scales.data_ptr(), offsets.data_ptr(), _ptr(rows),
                                T, E, N, K, out.data_ptr(), flags, _stream()))
    return out


# ---- the integer form of the 8-bit layers: codes (torch.int8) with a float32 scale per row: per token of the activations (codes [M,K], scales [M]), per channel of
# the weights (codes [N,K], scales [N], or with experts in front).  These calls and the router's take their tensors from the current device.
INT8_MAX_K = 131056


def _new(like, shape, dtype):
    return (like.new_empty if type(like) is _Tensor else _plain_empty(like))(shape, dtype=dtype)


def _is_tensor(t, dtype, *shape):
    """A contiguous tensor on the current device."""
    assert t.is_cuda and t.device.index == _current_device() and t.dtype == dtype and t.is_contiguous() and tuple(t.shape) == shape


def _is_operand8i(codes, scales, *shape):
    _is_tensor(codes, torch.int8, *shape)
    _is_tensor(scales, torch.float32, *shape[:-1])


def int8_rmsnorm_quantize(x, weight, eps: float = 1e-6, *, residual=None, residual_out=None, norm_out=None, codes=None, scales=None):
    """codes, scales, h = Q(v) with v = h * weight / sqrt(mean(h^2) + eps) and h = bf16(x + residual), or x (then the third result is None).
    x: bf16 [M,K], rows may be apart (K % 16 == 0, K <= 65536); weight: bf16 [K]; residual: bf16 [M,K].  residual_out: where h goes (may be residual
    or x themselves, a new tensor if None); norm_out: bf16 [M,K] to receive v too."""
    if _calls is not None and residual_out is None and codes is None and scales is None:
        out = _calls.rmsnorm_quantize8i(x, weight, eps, residual, norm_out)
        if out is not None:
            return out
    M, K, stride = _rows(x)
    assert x.device.index == _current_device()
    _is_tensor(weight, torch.bfloat16, K)
    if residual is not None and residual_out is None:
        residual_out = _new(x, (M, K), torch.bfloat16)
    for t in (residual, residual_out, norm_out):
        if t is not None:
            _is_tensor(t, torch.bfloat16, M, K)
    codes = _new(x, (M, K), torch.int8) if codes is None else codes
    scales = _new(x, (M,), torch.float32) if scales is None else scales
    _is_operand8i(codes, scales, M, K)
    _check(lib.int8_rmsnorm_quantize(x.data_ptr(), stride, _ptr(residual), weight.data_ptr(), M, K, eps, codes.data_ptr(), scales.data_ptr(), _ptr(residual_out),
                                     _ptr(norm_out), 0, _stream()))
    return codes, scales, residual_out


def int8_quantize(x, *, flags: int = 0, codes=None, scales=None):
    """codes, scales = Q(x), a scale per row, of bf16 activations [M,K] (rows may be apart), or with SILU_MUL of silu(x[:, :K]) * x[:, K:] of x [M, 2K]; of weights [N,K], or of
    experts [E,N,K] (contiguous).  K % 16 == 0."""
    if _calls is not None and codes is None and scales is None:
        out = _calls.quantize8i(x, flags)
        if out is not None:
            return out
    if x.dim() == 3:
        assert x.is_cuda and x.dtype == torch.bfloat16 and x.is_contiguous()
        M, K, stride = x.shape[0] * x.shape[1], x.shape[2], x.shape[2]
    else:
        M, K, stride = _rows(x)
    assert x.device.index == _current_device()
    if flags & SILU_MUL:
        assert K % 2 == 0
        K //= 2
    shape = (*x.shape[:-1], K)
    codes = _new(x, shape, torch.int8) if codes is None else codes
    scales = _new(x, shape[:-1], torch.float32) if scales is None else scales
    _is_operand8i(codes, scales, *shape)
    _check(lib.int8_quantize(x.data_ptr(), stride, M, K, codes.data_ptr(), scales.data_ptr(), flags, _stream()))
    return codes, scales


def _product8i_out(a_codes, a_scales, w_codes, w_scales, dim: int, rows: int, flags: int, out):
    assert a_codes.dim() == 2 and w_codes.dim() == dim
    N, K = w_codes.shape[-2:]
    _is_operand8i(a_codes, a_scales, a_codes.shape[0], K)
    _is_operand8i(w_codes, w_scales, *w_codes.shape)
    dtype = torch.float32 if flags & OUT_F32 else torch.bfloat16
    out = _new(a_codes, (rows, N), dtype) if out is None else out
    _is_tensor(out, dtype, rows, N)
    return out, N, K


def int8_gemm(a_codes, a_scales, w_codes, w_scales, *, flags: int = 0, out=None, workspace=None):
    """out[M,N] = A W^T (bf16, or fp32 with OUT_F32) from the int8 codes and row scales of activations [M,K] and weights [N,K]; the sums are exact."""
    if _calls is not None and out is None and workspace is None:
        got = _calls.gemm8i(a_codes, a_scales, w_codes, w_scales, flags)
        if got is not None:
            return got
    M = a_codes.shape[0]
    out, N, K = _product8i_out(a_codes, a_scales, w_codes, w_scales, 2, M, flags, out)
    need = int8_workspace_bytes(M, N, K)
    if need and workspace is None:
        workspace = _new(a_codes, (need,), torch.uint8)
    assert workspace is None or (workspace.is_cuda and workspace.device == a_codes.device and workspace.is_contiguous())
    wsz = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib.int8_gemm(a_codes.data_ptr(), a_scales.data_ptr(), w_codes.data_ptr(), w_scales.data_ptr(), M, N, K, out.data_ptr(), _ptr(workspace), wsz, flags, _stream()))
    return out


def int8_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(lib.int8_workspace_bytes(M, N, K))


def int8_grouped_gemm(a_codes, a_scales, w_codes, w_scales, offsets, *, rows=None, flags: int = 0, out=None):
    """Rows offsets[e] .. offsets[e+1] - 1 of out = those rows of A times the weights of expert e, w_codes [E,N,K]; offsets: int32 [E+1].
    rows: int32 [T], the row of A for each row of out (outside A: a row of zeros); without it out has A's rows.  Rows of out that no expert has are
    not written (a new out holds what its memory held)."""
    if _calls is not None and out is None:
        got = _calls.gemm8i(a_codes, a_scales, w_codes, w_scales, flags, offsets, rows)
        if got is not None:
            return got
    _is_tensor(offsets, torch.int32, w_codes.shape[0] + 1)
    T = a_codes.shape[0]
    if rows is not None:
        T = rows.shape[0]
        _is_tensor(rows, torch.int32, T)
    out, N, K = _product8i_out(a_codes, a_scales, w_codes, w_scales, 3, T, flags, out)
    _check(lib.int8_grouped_gemm(a_codes.data_ptr(), a_scales.data_ptr(), a_codes.shape[0], w_codes.data_ptr(), w_scales.data_ptr(), offsets.data_ptr(), _ptr(rows),
                                 T, w_codes.shape[0], N, K, out.data_ptr(), flags, _stream()))
    return out


# ---- a router's choice of experts, and their outputs added up
def moe_workspace_bytes(T: int, experts: int, top: int) -> int:
    return int(lib.moe_workspace_bytes(T, experts, top))


def moe_route(logits, top: int, *, bias=None, groups: int = 1, top_groups: int = 1, scale: float = 1.0, flags: int = 0, workspace=None):
    """weights, experts, rows, offsets, places from the logits [T,E] of a router (bf16 or float32; rows may be apart): each token's `top` best experts (int32 [T,top], in descending
    order, equal ones by index) and their weights (float32), and the rows by expert that the grouped products take: the token of each row (int32 [T*top]), where each expert's begin
    (int32 [E+1]), and each choice's row (int32 [T,top]).  flags: ROUTE_SIGMOID (scores; else softmax), ROUTE_RENORM (weights divided by their sum), ROUTE_GROUP_SUM2.  bias: float32 [E],
    added to the scores for the choice alone.  groups, top_groups: only the experts of the best groups may be chosen.  An expert of -inf is not chosen; a choice that a token does
    not have is -1, with a weight of 0 and a place of -1, and has no row (rows behind offsets[E] are not written)."""
    if _calls is not None and workspace is None:
        got = _calls.route(logits, top, bias, groups, top_groups, scale, flags)
        if got is not None:
            return got
    assert logits.is_cuda and logits.device.index == _current_device() and logits.dim() == 2 and logits.dtype in (torch.bfloat16, torch.float32)
    T, E = logits.shape
    assert logits.stride(1) == 1 or E <= 1
    stride = logits.stride(0) if T > 1 else E
    assert logits.dtype == torch.float32 or not flags & INPUT_F32
    if logits.dtype == torch.float32:
        flags |= INPUT_F32
    if bias is not None:
        _is_tensor(bias, torch.float32, E)
    assert 0 < top <= E
    weights, experts, places = _new(logits, (T, top), torch.float32), _new(logits, (T, top), torch.int32), _new(logits, (T, top), torch.int32)
    rows, offsets = _new(logits, (T * top,), torch.int32), _new(logits, (E + 1,), torch.int32)
    need = moe_workspace_bytes(T, E, top)
    if need and workspace is None:
        workspace = _new(logits, (need,), torch.uint8)
    assert workspace is None or (workspace.is_cuda and workspace.device == logits.device and workspace.is_contiguous())
    wsz = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib.moe_route(logits.data_ptr(), stride, _ptr(bias), T, E, top, groups, top_groups, scale, weights.data_ptr(), experts.data_ptr(), rows.data_ptr(), offsets.data_ptr(),
                         places.data_ptr(), _ptr(workspace), wsz, flags, _stream()))
    return weights, experts, rows, offsets, places


def moe_combine(y, places, weights, *, shared=None, flags: int = 0, out=None):
    """out[T,H] = shared + sum over j of weights[:, j] * y[places[:, j]], in float32 and rounded once (bf16, or float32 with OUT_F32).  y: bf16 or float32 [rows,H]; places: int32 [T,top]
    (outside y: the weight times zero); weights: float32 [T,top]; shared: bf16 or float32 [T,H] (may be out)."""
    if _calls is not None and out is None:
        got = _calls.combine(y, places, weights, shared, flags)
        if got is not None:
            return got
    assert y.dim() == 2 and places.dim() == 2 and y.dtype in (torch.bfloat16, torch.float32)
    R, H = y.shape
    T, top = places.shape
    _is_tensor(y, y.dtype, R, H)
    _is_tensor(places, torch.int32, T, top)
    _is_tensor(weights, torch.float32, T, top)
    assert y.dtype == torch.float32 or not flags & INPUT_F32
    if y.dtype == torch.float32:
        flags |= INPUT_F32
    assert not flags & SHARED_F32 or (shared is not None and shared.dtype == torch.float32)
    if shared is not None:
        assert shared.dtype in (torch.bfloat16, torch.float32)
        _is_tensor(shared, shared.dtype, T, H)
        if shared.dtype == torch.float32:
            flags |= SHARED_F32
    dtype = torch.float32 if flags & OUT_F32 else torch.bfloat16
    out = _new(y, (T, H), dtype) if out is None else out
    _is_tensor(out, dtype, T, H)
    _check(lib.moe_combine(y.data_ptr(), R, places.data_ptr(), weights.data_ptr(), _ptr(shared), T, top, H, out.data_ptr(), flags, _stream()))
    return out


def set_option(option: int, value: int) -> None:
    """Process-wide tuning / cross-check switch (OPT_GEMM_VARIANT, OPT_GEMM_GRID, OPT_SW_CODEC, OPT_FP8_VARIANT, OPT_INT8_VARIANT); 0 restores the default."""
    _check(lib.fp4_set_option(int(option), int(value)))


def version() -> int:
    return int(lib.fp4_version())
