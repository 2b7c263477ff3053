"""CPU-only checks of the low-precision operators: what the library refuses before it would touch a GPU, and what the
Python binding refuses."""

import ctypes as C

import pytest

torch = pytest.importorskip("torch")
import paper_1811_10751_b200 as g            # noqa: E402

P = C.c_void_p(4096)                          # never dereferenced: the checks come first
L = g.lib


def test_norm_argument_checks():
    def call(type_=1, x=P, ldx=256, res=None, ldr=0, wtype=1, w=P, h=None, ldh=0, q=None, ldq=0, sc=None, lds=0, T=4, H=256, qt=3):
        return L.gpd_rmsnorm_quant(type_, x, ldx, res, ldr, wtype, w, 1e-5, h, ldh, None, 0, qt, q, ldq, sc, lds, None, T, H, None)
    assert call(type_=3) == g.GPD_ERR_ARG and call(wtype=2) == g.GPD_ERR_ARG and call(x=None) == g.GPD_ERR_ARG
    assert call(w=None) == g.GPD_ERR_ARG and call(q=P, ldq=256) == g.GPD_ERR_ARG
    assert call(q=P, ldq=256, sc=P, lds=2, qt=1) == g.GPD_ERR_ARG
    assert call(H=0) == g.GPD_ERR_SHAPE and call(T=-1) == g.GPD_ERR_SHAPE and call(ldx=255) == g.GPD_ERR_SHAPE
    assert call(res=P, ldr=255) == g.GPD_ERR_SHAPE and call(h=P, ldh=1) == g.GPD_ERR_SHAPE
    assert call(q=P, ldq=255, sc=P, lds=2) == g.GPD_ERR_SHAPE and call(q=P, ldq=256, sc=P, lds=1) == g.GPD_ERR_SHAPE
    assert call(T=0, x=None) == g.GPD_OK      # empty buffers may have no address

    def back(dw=P, ws=P, n=4 * 256 * 4, dx=P, T=4):
        return L.gpd_rmsnorm_backward(1, P, 256, P, 256, 1, P, P, None, 0, dx, 256, dw, T, 256, ws, n, None)
    assert back(dw=None) == g.GPD_ERR_ARG and back(dx=None) == g.GPD_ERR_ARG
    assert back(ws=None) == g.GPD_ERR_WORKSPACE and back(n=4 * 256 * 4 - 1) == g.GPD_ERR_WORKSPACE
    assert back(T=-1) == g.GPD_ERR_SHAPE


def test_cut_and_product_argument_checks():
    def cut(type_=1, qt=3, br=1, q=P, ldq=256, s=P, lds=2, M=4, K=256, ld=256, src=P):
        return L.gpd_quantize_blocks(type_, src, ld, qt, br, q, ldq, s, lds, None, 0, None, 0, M, K, None)
    assert cut(type_=4) == g.GPD_ERR_ARG and cut(qt=0) == g.GPD_ERR_ARG and cut(br=2) == g.GPD_ERR_ARG
    assert cut(q=None) == g.GPD_ERR_ARG and cut(s=None) == g.GPD_ERR_ARG and cut(src=None) == g.GPD_ERR_ARG
    assert cut(ld=255) == g.GPD_ERR_SHAPE and cut(ldq=255) == g.GPD_ERR_SHAPE and cut(lds=1) == g.GPD_ERR_SHAPE
    assert cut(M=-1) == g.GPD_ERR_SHAPE and cut(M=0, src=None, q=None) == g.GPD_OK

    def mul(at=3, A=P, lda=256, sa=P, ldsa=2, ar=1, bt=3, ot=1, D=P, ldd=8, M=4, N=8, K=256, br=128):
        return L.gpd_gemm_fp8(at, A, lda, sa, ldsa, ar, bt, P, 256, P, 2, br, ot, D, ldd, M, N, K, 0, None)
    assert mul(at=1) == g.GPD_ERR_ARG and mul(bt=0) == g.GPD_ERR_ARG and mul(ot=3) == g.GPD_ERR_ARG
    assert mul(ar=64) == g.GPD_ERR_ARG and mul(br=0) == g.GPD_ERR_ARG and mul(A=None) == g.GPD_ERR_ARG and mul(D=None) == g.GPD_ERR_ARG
    assert mul(A=C.c_void_p(4104)) == g.GPD_ERR_ARG and mul(lda=264) == g.GPD_ERR_ARG          # 16-byte boundaries
    assert mul(lda=240) == g.GPD_ERR_SHAPE and mul(ldsa=1) == g.GPD_ERR_SHAPE and mul(ldd=7) == g.GPD_ERR_SHAPE
    assert mul(K=-1) == g.GPD_ERR_SHAPE and mul(M=0, D=None) == g.GPD_OK and mul(K=1 << 31) == g.GPD_ERR_SHAPE


def test_logit_argument_checks():
    def logp(type_=1, x=P, ld=100, ib=4, tok=P, G=1, tau=1.0, lp=P, lse=P, K=0, ids=None, T=2, V=100):
        return L.gpd_token_logprobs(type_, x, ld, ib, tok, G, tau, lp, lse, None, K, ids, None, T, V, None)
    assert logp(type_=3) == g.GPD_ERR_ARG and logp(tau=0.0) == g.GPD_ERR_ARG and logp(tau=float("nan")) == g.GPD_ERR_ARG
    assert logp(lse=None) == g.GPD_ERR_ARG and logp(tok=None) == g.GPD_ERR_ARG and logp(ib=2) == g.GPD_ERR_ARG and logp(K=3) == g.GPD_ERR_ARG
    assert logp(ld=99) == g.GPD_ERR_SHAPE and logp(G=65) == g.GPD_ERR_SHAPE and logp(K=33, ids=P) == g.GPD_ERR_SHAPE
    assert logp(V=5, K=6, ids=P) == g.GPD_ERR_SHAPE and logp(V=0) == g.GPD_ERR_SHAPE and logp(T=0, x=None) == g.GPD_OK

    def back(H=None, gh=None, d=P, ldd=100, tau=1.0):
        return L.gpd_token_logprobs_backward(1, P, 100, 4, P, 1, tau, P, H, P, gh, d, ldd, 2, 100, None)
    assert back(gh=P) == g.GPD_ERR_ARG and back(d=None) == g.GPD_ERR_ARG and back(ldd=99) == g.GPD_ERR_SHAPE and back(tau=-1.0) == g.GPD_ERR_ARG

    def dist(ids=P, ldi=8, tt=0, t=P, K=8, loss=P, ib=4, d=None, ldd=0, V=100):
        return L.gpd_distill_topk(1, P, V, ib, ids, ldi, tt, t, 8, K, None, 1.0, loss, d, ldd, 2, V, None)
    assert dist(ids=None) == g.GPD_ERR_ARG and dist(t=None) == g.GPD_ERR_ARG and dist(loss=None) == g.GPD_ERR_ARG and dist(ib=1) == g.GPD_ERR_ARG
    assert dist(tt=4) == g.GPD_ERR_ARG and dist(K=1025) == g.GPD_ERR_SHAPE and dist(ldi=7) == g.GPD_ERR_SHAPE and dist(d=P, ldd=99) == g.GPD_ERR_SHAPE


def test_binding_refuses_host_tensors_and_wrong_ranks():
    x, w = torch.zeros((2, 64)), torch.ones(64)
    with pytest.raises(ValueError, match="device tensor"):
        g.gpd_rmsnorm_quant(x, w, 1e-5, y=x)
    with pytest.raises(ValueError, match="device tensor"):
        g.gpd_quantize_blocks(x, q=x, scales=x)
    with pytest.raises(ValueError, match="device tensor"):
        g.gpd_gemm_fp8(x, x, x, x, x)
    with pytest.raises(ValueError, match="device tensor"):
        g.gpd_token_logprobs(x, w, w, w)
    with pytest.raises(ValueError, match="tensor expected"):
        g.gpd_distill_topk(None, x, x, None, w)


def test_new_fp8_rows_start_where_the_product_wants_them():
    for rows, cols, br in ((3, 100, 1), (130, 4100, 128), (1, 1, 1), (5, 0, 1)):
        q, s = g.new_fp8(rows, cols, block_rows=br, device="cpu")
        assert q.shape == (rows, cols) and q.stride(0) % 16 == 0 and q.data_ptr() % 16 == 0
        assert s.shape == (-(-rows // br), -(-cols // 128)) and s.stride(0) % 4 == 0
