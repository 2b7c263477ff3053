"""Binding of the low-precision layer and output-head operators (last section of include/gpd.h).

Tensors are two-dimensional [rows, columns] with unit column stride and any row stride; types are FP32,
BF16 or FP16, 8-bit values torch.float8_e4m3fn or torch.float8_e5m2, block scales torch.float8_e8m0fnu
(or uint8 holding the same bytes).  Outputs are buffers of the caller's; `new_fp8` makes the 8-bit ones.
Wrong devices, types, shapes or strides raise ValueError here, what the library refuses raises GpdError.
"""

from __future__ import annotations

import ctypes as C
from typing import Optional

import torch

from .binding import EXPORTED, _check, lib

GPD_DT_F32, GPD_DT_BF16, GPD_DT_F16, GPD_DT_E4M3, GPD_DT_E5M2 = range(5)
GPD_RMSNORM_MAX_PARTS = 512
GPD_LOGPROBS_MAX_TOP, GPD_LOGPROBS_MAX_TOKENS, GPD_DISTILL_MAX_TOP = 32, 64, 1024
_DT = {torch.float32: GPD_DT_F32, torch.bfloat16: GPD_DT_BF16, torch.float16: GPD_DT_F16,
       torch.float8_e4m3fn: GPD_DT_E4M3, torch.float8_e5m2: GPD_DT_E5M2}
_FLOATS = (torch.float32, torch.bfloat16, torch.float16)
_FP8 = (torch.float8_e4m3fn, torch.float8_e5m2)
_SCALES = (torch.float8_e8m0fnu, torch.uint8)
_F32 = (torch.float32,)
_I32 = (torch.int32,)
_INDEX = (torch.int32, torch.int64)
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


def _where(device: torch.device, stream) -> int:
    """Stream handle for work on tensors of `device`, which has to be the current device."""
    if device.type != "cuda":
        raise ValueError("device tensor expected")
    if device.index != torch.cuda.current_device():
        raise ValueError(f"tensors are on {device}, the current device is cuda:{torch.cuda.current_device()}")
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(device.index)
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _mat(name: str, t: Optional[torch.Tensor], device, dtypes, rows: int, cols: int):
    """(pointer, row stride) of a [rows, cols] matrix; (None, 0) if there is none."""
    if t is None:
        return None, 0
    if t.dtype not in dtypes:
        raise ValueError(f"{name}: tensor of {' or '.join(map(str, dtypes))} expected, got {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name}: tensor on {device} expected, got {t.device}")
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] != cols:
        raise ValueError(f"{name}: shape ({rows}, {cols}) expected, got {tuple(t.shape)}")
    sr, sc = t.stride()
    if sc != 1 and cols > 1:
        raise ValueError(f"{name}: columns have to be adjacent (stride {t.stride()})")
    if sr < cols:
        if rows > 1:
            raise ValueError(f"{name}: rows overlap (stride {t.stride()})")
        sr = cols
    return t.data_ptr(), sr


def _vec(name: str, t: Optional[torch.Tensor], device, dtypes, n: int):
    if t is None:
        return None
    if t.dtype not in dtypes:
        raise ValueError(f"{name}: tensor of {' or '.join(map(str, dtypes))} expected, got {t.dtype}")
    if t.device != device or t.dim() != 1 or t.shape[0] != n or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{name}: contiguous vector of {n} on {device} expected, got {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _rank2(name: str, t: torch.Tensor):
    if t.dim() != 2:
        raise ValueError(f"{name}: matrix expected, got shape {tuple(t.shape)}")
    return t.shape


def _blocks(n: int, per: int = _BLOCK) -> int:
    return (n + per - 1) // per


def new_fp8(rows: int, cols: int, dtype: torch.dtype = torch.float8_e4m3fn, block_rows: int = 1, device="cuda"):
    """Uninitialised 8-bit matrix and its block scales, with the row strides gpd_gemm_fp8 wants (multiples of
    16 and 4 bytes): (q [rows, cols], scales [ceil(rows / block_rows), ceil(cols / 128)])."""
    q = torch.empty((rows, max(16, _blocks(cols, 16) * 16)), dtype=dtype, device=device)[:, :cols]
    kb = _blocks(cols)
    s = torch.empty((_blocks(rows, block_rows), max(4, _blocks(kb, 4) * 4)), dtype=torch.float8_e8m0fnu, device=device)
    return q, s[:, :kb]


def gpd_rmsnorm_quant(x, weight, eps: float, residual=None, residual_out=None, y=None, q=None, scales=None, rstd=None,
                      stream=None):
    T, H = _rank2("x", x)
    dev, dt = x.device, x.dtype
    st = _where(dev, stream)
    if dt not in _FLOATS:
        raise ValueError(f"x: FP32, BF16 or FP16 expected, got {dt}")
    same = (dt,)
    px, ldx = _mat("x", x, dev, same, T, H)
    pr, ldr = _mat("residual", residual, dev, same, T, H)
    pw = _vec("weight", weight, dev, (dt, torch.float32), H)
    ph, ldh = _mat("residual_out", residual_out, dev, same, T, H)
    py, ldy = _mat("y", y, dev, same, T, H)
    pq, ldq = _mat("q", q, dev, _FP8, T, H)
    if q is not None and scales is None:
        raise ValueError("scales: needed with q")
    ps, lds = _mat("scales", scales, dev, _SCALES, T, _blocks(H))
    _check(lib.gpd_rmsnorm_quant(_DT[dt], px, ldx, pr, ldr, _DT[weight.dtype], pw, eps, ph, ldh, py, ldy,
                                 GPD_DT_E4M3 if q is None else _DT[q.dtype], pq, ldq, ps, lds,
                                 _vec("rstd", rstd, dev, _F32, T), T, H, st), "gpd_rmsnorm_quant")


def gpd_rmsnorm_backward(dy, h, weight, rstd, dx, dweight, workspace, dresidual=None, stream=None):
    """workspace: at least min(T, GPD_RMSNORM_MAX_PARTS) * H floats of any type, contiguous."""
    T, H = _rank2("h", h)
    dev, dt = h.device, h.dtype
    st = _where(dev, stream)
    if dt not in _FLOATS:
        raise ValueError(f"h: FP32, BF16 or FP16 expected, got {dt}")
    same = (dt,)
    py, lddy = _mat("dy", dy, dev, same, T, H)
    ph, ldh = _mat("h", h, dev, same, T, H)
    pd, lddh = _mat("dresidual", dresidual, dev, same, T, H)
    px, lddx = _mat("dx", dx, dev, same, T, H)
    if workspace.device != dev or not workspace.is_contiguous():
        raise ValueError(f"workspace: contiguous buffer on {dev} expected")
    _check(lib.gpd_rmsnorm_backward(_DT[dt], py, lddy, ph, ldh, _DT[weight.dtype],
                                    _vec("weight", weight, dev, (dt, torch.float32), H), _vec("rstd", rstd, dev, _F32, T),
                                    pd, lddh, px, lddx, _vec("dweight", dweight, dev, _F32, H), T, H,
                                    workspace.data_ptr(), workspace.numel() * workspace.element_size(), st),
           "gpd_rmsnorm_backward")


def gpd_quantize_blocks(src, q=None, scales=None, qT=None, scalesT=None, block_rows: int = 1, stream=None):
    M, K = _rank2("src", src)
    dev = src.device
    st = _where(dev, stream)
    if src.dtype not in _FLOATS:
        raise ValueError(f"src: FP32, BF16 or FP16 expected, got {src.dtype}")
    if block_rows not in (1, _BLOCK):
        raise ValueError("block_rows: 1 or 128")
    if q is None and qT is None:
        raise ValueError("q or qT: one of them is needed")
    if (q is None) != (scales is None) or (qT is None) != (scalesT is None):
        raise ValueError("8-bit values and their scales go together")
    if q is not None and qT is not None and q.dtype != qT.dtype:
        raise ValueError("q and qT: one 8-bit type expected")
    ps, ld = _mat("src", src, dev, _FLOATS, M, K)
    pq, ldq = _mat("q", q, dev, _FP8, M, K)
    pqs, lds = _mat("scales", scales, dev, _SCALES, _blocks(M, block_rows), _blocks(K))
    pt, ldt = _mat("qT", qT, dev, _FP8, K, M)
    pts, ldts = _mat("scalesT", scalesT, dev, _SCALES, _blocks(K, block_rows), _blocks(M))
    _check(lib.gpd_quantize_blocks(_DT[src.dtype], ps, ld, _DT[(qT if q is None else q).dtype], block_rows, pq, ldq, pqs,
                                   lds, pt, ldt, pts, ldts, M, K, st), "gpd_quantize_blocks")


def _scale_rows(name: str, s, rows: int) -> int:
    """Operand rows that share a row of scales: 1 or 128, told from the number of scale rows."""
    if s.dim() == 2 and s.shape[0] == rows:
        return 1
    if s.dim() == 2 and s.shape[0] == _blocks(rows):
        return _BLOCK
    raise ValueError(f"{name}: {rows} or {_blocks(rows)} rows of scales expected, got shape {tuple(s.shape)}")


def gpd_gemm_fp8(A, a_scales, B, b_scales, out, accumulate: bool = False, stream=None):
    """out (M x N) = A (M x K) B (N x K)^T with block scales; one scale row per operand row or per 128 of them."""
    M, K = _rank2("A", A)
    N = _rank2("B", B)[0]
    dev = A.device
    st = _where(dev, stream)
    pa, lda = _mat("A", A, dev, _FP8, M, K)
    pb, ldb = _mat("B", B, dev, _FP8, N, K)
    ra, rb, kb = _scale_rows("a_scales", a_scales, M), _scale_rows("b_scales", b_scales, N), _blocks(K)
    psa, ldsa = _mat("a_scales", a_scales, dev, _SCALES, a_scales.shape[0], kb)
    psb, ldsb = _mat("b_scales", b_scales, dev, _SCALES, b_scales.shape[0], kb)
    po, ldd = _mat("out", out, dev, _FLOATS, M, N)
    if M == 1 and lda % 16:
        lda = _blocks(lda, 16) * 16                    # a single row has no stride
    if N == 1 and ldb % 16:
        ldb = _blocks(ldb, 16) * 16
    _check(lib.gpd_gemm_fp8(_DT[A.dtype], pa, lda, psa, ldsa, ra, _DT[B.dtype], pb, ldb, psb, ldsb, rb, _DT[out.dtype], po,
                            ldd, M, N, K, accumulate, st), "gpd_gemm_fp8")


def _per_row(name: str, t, device, dtypes, T: int, G: int):
    """Pointer of a contiguous [T] (G = 1) or [T, G] tensor."""
    if t is None:
        return None
    if t.dtype not in dtypes:
        raise ValueError(f"{name}: tensor of {' or '.join(map(str, dtypes))} expected, got {t.dtype}")
    if t.device != device or t.dim() not in (1, 2) or t.numel() != T * G or t.shape[0] != T or not t.is_contiguous():
        raise ValueError(f"{name}: contiguous ({T}, {G}) tensor on {device} expected, got {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _tokens_per_row(tokens, T: int) -> int:
    if tokens.dim() == 1:
        return 1
    if tokens.dim() == 2:
        return tokens.shape[1]
    raise ValueError(f"tokens: [T] or [T, G] expected, got shape {tuple(tokens.shape)}")


def gpd_token_logprobs(logits, tokens, logprobs, lse, entropy=None, top_ids=None, top_logprobs=None,
                       temperature: float = 1.0, stream=None):
    """tokens, logprobs: [T] or [T, G]; top_ids (int32), top_logprobs: [T, K]."""
    T, V = _rank2("logits", logits)
    dev = logits.device
    st = _where(dev, stream)
    px, ld = _mat("logits", logits, dev, _FLOATS, T, V)
    G = _tokens_per_row(tokens, T)
    K = 0
    if top_ids is not None:
        K = _rank2("top_ids", top_ids)[1]
    elif top_logprobs is not None:
        raise ValueError("top_ids: needed with top_logprobs")
    if lse is None:
        raise ValueError("lse: needed")
    _check(lib.gpd_token_logprobs(_DT[logits.dtype], px, ld, tokens.element_size(),
                                  _per_row("tokens", tokens, dev, _INDEX, T, G), G, temperature,
                                  _per_row("logprobs", logprobs, dev, _F32, T, G), _vec("lse", lse, dev, _F32, T),
                                  _vec("entropy", entropy, dev, _F32, T), K, _per_row("top_ids", top_ids, dev, _I32, T, K),
                                  _per_row("top_logprobs", top_logprobs, dev, _F32, T, K), T, V, st), "gpd_token_logprobs")


def gpd_token_logprobs_backward(logits, tokens, lse, entropy, dlogprobs, dentropy, dlogits, temperature: float = 1.0,
                                stream=None):
    """dlogprobs, dentropy: upstream gradients, either may be None; entropy is needed with dentropy."""
    T, V = _rank2("logits", logits)
    dev = logits.device
    st = _where(dev, stream)
    px, ld = _mat("logits", logits, dev, _FLOATS, T, V)
    pd, ldd = _mat("dlogits", dlogits, dev, (logits.dtype,), T, V)
    G = _tokens_per_row(tokens, T)
    _check(lib.gpd_token_logprobs_backward(_DT[logits.dtype], px, ld, tokens.element_size(),
                                           _per_row("tokens", tokens, dev, _INDEX, T, G), G, temperature,
                                           _vec("lse", lse, dev, _F32, T), _vec("entropy", entropy, dev, _F32, T),
                                           _per_row("dlogprobs", dlogprobs, dev, _F32, T, G),
                                           _vec("dentropy", dentropy, dev, _F32, T), pd, ldd, T, V, st),
           "gpd_token_logprobs_backward")


def gpd_distill_topk(logits, teacher_ids, teacher_logits, weights, loss, dlogits=None, temperature: float = 1.0, stream=None):
    """teacher_ids, teacher_logits: [T, K]; weights: [T] or None; dlogits: None for the loss alone."""
    T, V = _rank2("logits", logits)
    K = _rank2("teacher_ids", teacher_ids)[1]
    dev = logits.device
    st = _where(dev, stream)
    px, ld = _mat("logits", logits, dev, _FLOATS, T, V)
    pi, ldi = _mat("teacher_ids", teacher_ids, dev, _INDEX, T, K)
    pt, ldt = _mat("teacher_logits", teacher_logits, dev, _FLOATS, T, K)
    pd, ldd = _mat("dlogits", dlogits, dev, (logits.dtype,), T, V)
    _check(lib.gpd_distill_topk(_DT[logits.dtype], px, ld, teacher_ids.element_size(), pi, ldi, _DT[teacher_logits.dtype], pt,
                                ldt, K, _vec("weights", weights, dev, _F32, T), temperature, _vec("loss", loss, dev, _F32, T),
                                pd, ldd, T, V, st), "gpd_distill_topk")
