"""Binding of the low-precision layer and output-head operators (last section of include/gpd.h).

Tensors are two-dimensional [rows, columns] with unit column stride and any row stride; types are FP32,
BF16 or FP16, 8-bit values torch.float8_e4m3fn or torch.float8_e5m2, block scales torch.float8_e8m0fnu
(or uint8 holding the same bytes).  Outputs are buffers of the caller's; `new_fp8` makes the 8-bit ones.
Wrong devices, types, shapes or strides raise ValueError here, what the library refuses raises GpdError.
"""

from __future__ import annotations

import ctypes as C

import torch

from .binding import EXPORTED, _check, lib
try:
    from . import _lm                                   # compiled from csrc/lm_binding.cpp
except ImportError as e:
    class _NotBuilt:
        """Stands for the compiled part where it cannot be loaded: the coded products do not need it, every operator of
        this file fails with the reason."""

        def __init__(self, why):
            self._why = why

        def __getattr__(self, name):
            raise ImportError(f"{self._why}: build it with `python paper_1811_10751_b200/build.py`. "
                              "This package has no CPU fallback.")

    _lm = _NotBuilt(str(e))

GPD_DT_F32, GPD_DT_BF16, GPD_DT_F16, GPD_DT_E4M3, GPD_DT_E5M2 = range(5)
GPD_RMSNORM_MAX_PARTS = 512
GPD_LOGPROBS_MAX_TOP, GPD_LOGPROBS_MAX_TOKENS, GPD_DISTILL_MAX_TOP = 32, 64, 1024
_BLOCK = 128

_vp, _i32, _i64, _f, _e = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_int
lib.gpd_rmsnorm_quant.argtypes = [_e, _vp, _i64, _vp, _i64, _e, _vp, _f, _vp, _i64, _vp, _i64, _e, _vp, _i64, _vp, _i64,
                                  _vp, _i64, _i64, _vp]
lib.gpd_rmsnorm_backward.argtypes = [_e, _vp, _i64, _vp, _i64, _e, _vp, _vp, _vp, _i64, _vp, _i64, _vp, _i64, _i64, _vp,
                                     _i64, _vp]
lib.gpd_quantize_blocks.argtypes = [_e, _vp, _i64, _e, _i32, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _i64, _i64, _vp]
lib.gpd_gemm_fp8.argtypes = [_e, _vp, _i64, _vp, _i64, _i32, _e, _vp, _i64, _vp, _i64, _i32, _e, _vp, _i64, _i64, _i64,
                             _i64, _i32, _vp]
lib.gpd_token_logprobs.argtypes = [_e, _vp, _i64, _i32, _vp, _i32, _f, _vp, _vp, _vp, _i32, _vp, _vp, _i64, _i64, _vp]
lib.gpd_token_logprobs_backward.argtypes = [_e, _vp, _i64, _i32, _vp, _i32, _f, _vp, _vp, _vp, _vp, _vp, _i64, _i64, _i64,
                                            _vp]
lib.gpd_distill_topk.argtypes = [_e, _vp, _i64, _i32, _vp, _i64, _e, _vp, _i64, _i32, _vp, _f, _vp, _vp, _i64, _i64, _i64,
                                 _vp]
_NAMES = ["gpd_rmsnorm_quant", "gpd_rmsnorm_backward", "gpd_quantize_blocks", "gpd_gemm_fp8", "gpd_token_logprobs",
          "gpd_token_logprobs_backward", "gpd_distill_topk"]
for _name in _NAMES:
    getattr(lib, _name).restype = C.c_int
EXPORTED += _NAMES


def _blocks(n: int, per: int = _BLOCK) -> int:
    return (n + per - 1) // per


def new_fp8(rows: int, cols: int, dtype: torch.dtype = torch.float8_e4m3fn, block_rows: int = 1, device="cuda"):
    """Uninitialised 8-bit matrix and its block scales: (q [rows, cols], scales [ceil(rows / block_rows), ceil(cols / 128)]).
    Rows start on 16-byte boundaries, as gpd_gemm_fp8 wants them, and on 128-byte ones from 128 columns on: a product
    of 4096 x 4096 x 4100 to FP32 with rows 4112 bytes apart takes 75 us, with rows 4224 bytes apart 64."""
    q = torch.empty((rows, max(16, _blocks(cols, 128) * 128 if cols >= 128 else _blocks(cols, 16) * 16)), dtype=dtype, device=device)
    kb = _blocks(cols)
    s = torch.empty((_blocks(rows, block_rows), max(4, _blocks(kb, 4) * 4)), dtype=torch.float8_e8m0fnu, device=device)
    return q[:, :cols], s[:, :kb]


def gpd_rmsnorm_quant(x, weight, eps: float, residual=None, residual_out=None, y=None, q=None, scales=None, rstd=None,
                      stream=None):
    status = _lm.rmsnorm_quant(x, weight, eps, residual, residual_out, y, q, scales, rstd, stream)
    if status:
        _check(status, "gpd_rmsnorm_quant")


def gpd_rmsnorm_backward(dy, h, weight, rstd, dx, dweight, workspace, dresidual=None, stream=None):
    """workspace: contiguous, at least min(T, GPD_RMSNORM_MAX_PARTS) * H * 4 bytes."""
    status = _lm.rmsnorm_backward(dy, h, weight, rstd, dx, dweight, workspace, dresidual, stream)
    if status:
        _check(status, "gpd_rmsnorm_backward")


def gpd_quantize_blocks(src, q=None, scales=None, qT=None, scalesT=None, block_rows: int = 1, stream=None):
    status = _lm.quantize_blocks(src, q, scales, qT, scalesT, block_rows, stream)
    if status:
        _check(status, "gpd_quantize_blocks")


def gpd_gemm_fp8(A, a_scales, B, b_scales, out, accumulate: bool = False, stream=None):
    """out (M x N) = A (M x K) B (N x K)^T with block scales; one scale row per operand row or per 128 of them, told
    from the number of scale rows."""
    status = _lm.gemm_fp8(A, a_scales, B, b_scales, out, accumulate, stream)
    if status:
        _check(status, "gpd_gemm_fp8")


def gpd_token_logprobs(logits, tokens, logprobs, lse, entropy=None, top_ids=None, top_logprobs=None,
                       temperature: float = 1.0, stream=None):
    """tokens, logprobs: [T] or [T, G]; top_ids (int32), top_logprobs: [T, K]."""
    status = _lm.token_logprobs(logits, tokens, logprobs, lse, entropy, top_ids, top_logprobs, temperature, stream)
    if status:
        _check(status, "gpd_token_logprobs")


def gpd_token_logprobs_backward(logits, tokens, lse, entropy, dlogprobs, dentropy, dlogits, temperature: float = 1.0,
                                stream=None):
    """dlogprobs, dentropy: upstream gradients, either may be None; entropy is needed with dentropy."""
    status = _lm.token_logprobs_backward(logits, tokens, lse, entropy, dlogprobs, dentropy, dlogits, temperature, stream)
    if status:
        _check(status, "gpd_token_logprobs_backward")


def gpd_distill_topk(logits, teacher_ids, teacher_logits, weights, loss, dlogits=None, temperature: float = 1.0, stream=None):
    """teacher_ids, teacher_logits: [T, K]; weights: [T] or None; dlogits: None for the loss alone."""
    status = _lm.distill_topk(logits, teacher_ids, teacher_logits, weights, loss, dlogits, temperature, stream)
    if status:
        _check(status, "gpd_distill_topk")
