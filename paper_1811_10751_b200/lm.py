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
GPD_HEAD_MAX_DIM, GPD_HEAD_MAX_AXES, GPD_HEAD_NORM_MAX_PARTS, GPD_GRAD_NORM_WORKSPACE = 256, 4, 512, 16384
GPD_ADAPTER_MAX_RANK = 128
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
lib.gpd_head_norm_rope.argtypes = [_e, _vp, _i64, _i32, _vp, _i64, _i32, _i32, _e, _vp, _vp, _f, _vp, _i64, _i64, _i32, _i32, _i32,
                                   _vp, _i64, _i32, _vp, _vp, _i64, _vp, _i64, _i64, _vp]
lib.gpd_head_norm_rope_backward.argtypes = [_e, _vp, _i64, _vp, _i64, _vp, _i64, _i32, _vp, _i64, _i32, _i32, _e, _vp, _vp, _f, _vp,
                                            _i64, _i64, _i32, _i32, _i32, _vp, _i64, _i32, _vp, _vp, _i64, _vp, _i64, _vp, _vp, _i64,
                                            _vp, _i64, _vp]
lib.gpd_grad_norm.argtypes = [_i32, _vp, _vp, _vp, _vp, _vp, _i64, _vp]
lib.gpd_clip_grads.argtypes = [_i32, _vp, _vp, _vp, _vp, _vp, _vp, _f, _vp]
lib.gpd_adapter.argtypes = [_e, _vp, _i64, _i32, _i32, _vp, _i64, _i64, _vp, _i64, _i64, _vp, _i32, _vp, _vp, _i32, _vp, _e, _vp, _i64,
                            _vp, _i64, _i64, _i64, _i64, _vp]
lib.gpd_adapter_backward_workspace.argtypes = [_i64, _i64, _i64, _i32, _i32, C.POINTER(_i64)]
lib.gpd_adapter_backward.argtypes = [_e, _vp, _i64, _vp, _i64, _i32, _i32, _vp, _i64, _i64, _vp, _i64, _i64, _vp, _vp, _i32, _vp, _vp,
                                     _i32, _e, _vp, _i64, _vp, _i64, _e, _vp, _i64, _i64, _vp, _i64, _i64, _i32, _i64, _i64, _i64,
                                     _vp, _i64, _vp]
_NAMES = ["gpd_rmsnorm_quant", "gpd_rmsnorm_backward", "gpd_quantize_blocks", "gpd_gemm_fp8", "gpd_token_logprobs",
          "gpd_token_logprobs_backward", "gpd_distill_topk", "gpd_head_norm_rope", "gpd_head_norm_rope_backward", "gpd_grad_norm",
          "gpd_clip_grads", "gpd_adapter", "gpd_adapter_backward_workspace", "gpd_adapter_backward"]
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


def new_rope_table(positions: int, rotated: int, base: float = 10000.0, device="cuda"):
    """Cosines and sines of the angles position * base^(-2 j / rotated) for gpd_head_norm_rope: [positions, rotated] FP32, pair
    j in columns j and rotated / 2 + j.  Angles are taken in FP64: far positions lose them in FP32."""
    j = torch.arange(rotated // 2, dtype=torch.float64, device=device)
    angle = torch.arange(positions, dtype=torch.float64, device=device)[:, None] * torch.pow(float(base), -2.0 * j / rotated)
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def gpd_head_norm_rope(q, k, table, positions, q_out, k_out, head_dim: int, q_weight=None, k_weight=None, eps: float = 1e-6,
                       axes=None, neighbours: bool = False, stream=None):
    """q, k: [T, heads * head_dim], either may be None with its output; table: [positions, rotated columns] FP32 or None for no
    rotation; positions: [T], or [T, axes] with axes (uint8, one for each pair); weights None: rotation alone."""
    status = _lm.head_norm_rope(q, k, table, positions, axes, q_out, k_out, head_dim, q_weight, k_weight, eps, neighbours, stream)
    if status:
        _check(status, "gpd_head_norm_rope")


def gpd_head_norm_rope_backward(dq, dk, q, k, table, positions, dq_in, dk_in, head_dim: int, q_weight=None, k_weight=None,
                                dq_weight=None, dk_weight=None, workspace=None, eps: float = 1e-6, axes=None,
                                neighbours: bool = False, stream=None):
    """dq, dk: gradients of the forward call's outputs; q, k: its inputs; dq_in, dk_in: theirs.  With weights: dq_weight,
    dk_weight ([head_dim] FP32) and workspace, 2 * GPD_HEAD_NORM_MAX_PARTS * head_dim * 4 bytes."""
    status = _lm.head_norm_rope_backward(dq, dk, table, positions, axes, q, k, dq_in, dk_in, head_dim, q_weight, k_weight, dq_weight,
                                         dk_weight, workspace, eps, neighbours, stream)
    if status:
        _check(status, "gpd_head_norm_rope_backward")


def gpd_grad_norm(grads, norm, workspace, stream=None):
    """grads: list of dense tensors, FP32, BF16 and FP16 mixed as they come; norm: [1] FP32; workspace:
    GPD_GRAD_NORM_WORKSPACE bytes."""
    status = _lm.grad_norm(grads, norm, workspace, stream)
    if status:
        _check(status, "gpd_grad_norm")


def gpd_clip_grads(grads, norm, max_norm: float, out=None, stream=None):
    """out: list of the gradients' shapes, of any of the three types; None: in place."""
    status = _lm.clip_grads(grads, norm, max_norm, out, stream)
    if status:
        _check(status, "gpd_clip_grads")


def gpd_adapter(x, A, B, offsets, index, out, h, base=None, scale=None, stream=None):
    """x: [T, K] BF16 or FP16; A: [adapters, rank, K], B: [adapters, N, rank] of its type; offsets: [S + 1], index: [S] (int32 or
    int64, -1: no adapter); out, base: [T, N] of x's type or FP32; h: [T, rank] FP32, kept for the backward call; scale: [adapters]
    FP32."""
    status = _lm.adapter(x, A, B, offsets, index, out, h, base, scale, stream)
    if status:
        _check(status, "gpd_adapter")


def gpd_adapter_backward_workspace(T: int, K: int, N: int, adapters: int, rank: int) -> int:
    """Bytes of workspace that gpd_adapter_backward needs for these sizes."""
    n = C.c_int64()
    _check(lib.gpd_adapter_backward_workspace(T, K, N, adapters, rank, C.byref(n)), "gpd_adapter_backward_workspace")
    return n.value


def gpd_adapter_backward(dout, x, A, B, h, offsets, index, dx, dA, dB, workspace, dbase=None, scale=None, accumulate: bool = False,
                         stream=None):
    """dx, dbase: [T, K] of x's type or FP32, dx may be None; dA, dB: the shapes of A and B, of x's type or FP32, both may be None;
    accumulate: dA and dB are added to."""
    status = _lm.adapter_backward(dout, x, A, B, h, offsets, index, dx, dA, dB, workspace, dbase, scale, accumulate, stream)
    if status:
        _check(status, "gpd_adapter_backward")
