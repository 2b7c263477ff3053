"""CPU-only checks of the adapter, head-norm and clipping operators: what the library refuses before it would touch a GPU."""

import ctypes as C
import math

import pytest

torch = pytest.importorskip("torch")
import paper_1811_10751_b200 as g            # noqa: E402

P = C.c_void_p(4096)                          # never dereferenced: the checks come first
L = g.lib


def test_head_argument_checks():
    def call(type_=1, q=P, ldq=256, Hq=2, k=P, ldk=128, Hk=1, D=128, wt=1, qw=P, kw=P, table=P, ldt=128, positions=10, R=128, ib=4, pos=P, ldp=1,
             axes=1, which=None, qo=P, ko=P, T=4):
        return L.gpd_head_norm_rope(type_, q, ldq, Hq, k, ldk, Hk, D, wt, qw, kw, 1e-6, table, ldt, positions, R, 0, ib, pos, ldp, axes, which, qo,
                                    256, ko, 128, T, None)
    assert call(type_=3) == g.GPD_ERR_ARG and call(wt=2) == g.GPD_ERR_ARG and call(q=None) == g.GPD_ERR_ARG and call(ko=None) == g.GPD_ERR_ARG
    assert call(qw=None) == g.GPD_ERR_ARG and call(ib=2) == g.GPD_ERR_ARG and call(table=None) == g.GPD_ERR_ARG and call(pos=None) == g.GPD_ERR_ARG
    assert call(axes=2, ldp=2) == g.GPD_ERR_ARG and call(qw=None, kw=None, R=0) == g.GPD_ERR_ARG
    assert call(D=0) == g.GPD_ERR_SHAPE and call(D=127) == g.GPD_ERR_SHAPE and call(D=258) == g.GPD_ERR_SHAPE and call(R=130) == g.GPD_ERR_SHAPE
    assert call(R=63) == g.GPD_ERR_SHAPE and call(ldq=255) == g.GPD_ERR_SHAPE and call(Hk=-1) == g.GPD_ERR_SHAPE and call(Hq=1025) == g.GPD_ERR_SHAPE
    assert call(axes=5, which=P) == g.GPD_ERR_SHAPE and call(ldt=127) == g.GPD_ERR_SHAPE and call(T=-1) == g.GPD_ERR_SHAPE
    assert call(T=0, q=None, k=None, pos=None) == g.GPD_OK and call(Hq=0, Hk=0) == g.GPD_OK

    def back(dq=P, q=P, dw=P, ws=P, n=2 * 512 * 128 * 4, T=4, w=P, lddq=256):
        return L.gpd_head_norm_rope_backward(1, dq, lddq, P, 128, q, 256, 2, P, 128, 1, 128, 1, w, w, 1e-6, P, 128, 10, 128, 0, 4, P, 1, 1, None, P, 256,
                                             P, 128, dw, P, T, ws, n, None)
    assert back(dq=None) == g.GPD_ERR_ARG and back(q=None) == g.GPD_ERR_ARG and back(dw=None) == g.GPD_ERR_ARG and back(lddq=255) == g.GPD_ERR_SHAPE
    assert back(ws=None) == g.GPD_ERR_WORKSPACE and back(n=2 * 512 * 128 * 4 - 1) == g.GPD_ERR_WORKSPACE
    assert back(T=0, w=None, dq=None) == g.GPD_OK


def test_gradient_list_argument_checks():
    def lists(ptrs, counts, types):
        n = len(ptrs)
        return n, (C.c_int32 * max(n, 1))(*types), (C.c_void_p * max(n, 1))(*ptrs), (C.c_int64 * max(n, 1))(*counts)

    def norm(ptrs=(4096,), counts=(8,), types=(0,), out=P, ws=P, size=g.GPD_GRAD_NORM_WORKSPACE, n=None):
        k, t, p, c = lists(ptrs, counts, types)
        return L.gpd_grad_norm(k if n is None else n, t, p, c, out, ws, size, None)
    assert norm(types=(3,)) == g.GPD_ERR_ARG and norm(ptrs=(None,)) == g.GPD_ERR_ARG and norm(ptrs=(4098,)) == g.GPD_ERR_ARG and norm(out=None) == g.GPD_ERR_ARG
    assert norm(counts=(-1,)) == g.GPD_ERR_SHAPE and norm(n=-1) == g.GPD_ERR_SHAPE and norm(counts=(1 << 46,)) == g.GPD_ERR_SHAPE
    assert norm(ws=None) == g.GPD_ERR_WORKSPACE and norm(size=g.GPD_GRAD_NORM_WORKSPACE - 1) == g.GPD_ERR_WORKSPACE
    assert norm(ws=C.c_void_p(4100)) == g.GPD_ERR_WORKSPACE
    assert L.gpd_grad_norm(1, None, None, None, P, P, g.GPD_GRAD_NORM_WORKSPACE, None) == g.GPD_ERR_ARG

    def clip(ptrs, outs, counts, types=None, out_types=None, bound=1.0, norm=P):
        n, t, p, c = lists(ptrs, counts, types or [0] * len(ptrs))
        _, ot, o, _ = lists(outs, counts, out_types or [0] * len(ptrs))
        return L.gpd_clip_grads(n, t, p, ot, o, c, norm, bound, None)
    for bad in (0.0, -1.0, math.nan):
        assert clip([4096], [4096], [8], bound=bad) == g.GPD_ERR_ARG
    assert clip([4096], [4096], [8], norm=None) == g.GPD_ERR_ARG and clip([4096], [4096], [8], out_types=[1]) == g.GPD_ERR_ARG
    assert clip([4096, 8192], [12288, 12288 + 28], [8, 8]) == g.GPD_ERR_ARG          # outputs overlap
    assert clip([4096, 8192], [12288, 4096], [8, 8]) == g.GPD_ERR_ARG                # an output over another's input
    assert clip([4096], [4096 + 16], [8]) == g.GPD_ERR_ARG and clip([4096, 4096], [4096, 4096], [8, 8]) == g.GPD_ERR_ARG
    assert clip([], [], []) == g.GPD_OK
    with pytest.raises(ValueError, match="device tensor"):
        g.gpd_grad_norm([torch.ones(3)], torch.ones(1), torch.ones(3))


def test_adapter_argument_checks():
    def call(type_=1, x=P, ldx=64, n=2, r=8, A=P, lda=64, na=512, B=P, ldb=8, nb=384, ib=4, off=P, idx=P, S=3, h=P, ot=1, base=None, ldbase=0, out=P,
             ldo=48, T=10, K=64, N=48):
        return L.gpd_adapter(type_, x, ldx, n, r, A, lda, na, B, ldb, nb, None, ib, off, idx, S, h, ot, base, ldbase, out, ldo, T, K, N, None)
    assert call(type_=0) == g.GPD_ERR_ARG and call(ot=2) == g.GPD_ERR_ARG and call(x=None) == g.GPD_ERR_ARG and call(h=None) == g.GPD_ERR_ARG
    assert call(out=None) == g.GPD_ERR_ARG and call(A=None) == g.GPD_ERR_ARG and call(off=None) == g.GPD_ERR_ARG and call(ib=1) == g.GPD_ERR_ARG
    assert call(r=0) == g.GPD_ERR_SHAPE and call(r=129, ldb=129) == g.GPD_ERR_SHAPE and call(ldx=63) == g.GPD_ERR_SHAPE and call(lda=63) == g.GPD_ERR_SHAPE
    assert call(na=511) == g.GPD_ERR_SHAPE and call(nb=383) == g.GPD_ERR_SHAPE and call(ldo=47) == g.GPD_ERR_SHAPE and call(K=0) == g.GPD_ERR_SHAPE
    assert call(base=P, ldbase=47) == g.GPD_ERR_SHAPE and call(S=-1) == g.GPD_ERR_SHAPE and call(T=1 << 31) == g.GPD_ERR_SHAPE
    assert call(T=0, x=None, out=None) == g.GPD_OK and call(S=0, off=None, idx=None) == g.GPD_OK

    size = C.c_int64()
    assert L.gpd_adapter_backward_workspace(10, 64, 48, 2, 8, C.byref(size)) == g.GPD_OK and size.value > 10 * 8 * 4
    assert L.gpd_adapter_backward_workspace(10, 64, 48, 2, 8, None) == g.GPD_ERR_ARG
    assert L.gpd_adapter_backward_workspace(-1, 64, 48, 2, 8, C.byref(size)) == g.GPD_ERR_SHAPE
    assert g.gpd_adapter_backward_workspace(10, 64, 48, 2, 8) == size.value

    def back(dout=P, x=P, h=P, dx=P, lddx=64, dA=P, dB=P, gt=0, ws=P, n=size.value, dbase=None, lddb=0):
        return L.gpd_adapter_backward(1, dout, 48, x, 64, 2, 8, P, 64, 512, P, 8, 384, None, h, 4, P, P, 3, 1, dbase, lddb, dx, lddx, gt, dA, 64, 512, dB, 8,
                                      384, 0, 10, 64, 48, ws, n, None)
    assert back(dout=None) == g.GPD_ERR_ARG and back(x=None) == g.GPD_ERR_ARG and back(h=None) == g.GPD_ERR_ARG and back(dA=None) == g.GPD_ERR_ARG
    assert back(gt=2) == g.GPD_ERR_ARG and back(lddx=63) == g.GPD_ERR_SHAPE and back(dbase=P, lddb=63) == g.GPD_ERR_SHAPE
    assert back(ws=None) == g.GPD_ERR_WORKSPACE and back(n=size.value - 1) == g.GPD_ERR_WORKSPACE and back(ws=C.c_void_p(4104)) == g.GPD_ERR_WORKSPACE
    assert back(dx=None, dA=None, dB=None) == g.GPD_OK


def test_table_of_angles():
    t = g.new_rope_table(100, 32, base=500.0, device="cpu")
    assert t.shape == (100, 32) and t.dtype == torch.float32
    for p, j in ((0, 0), (7, 3), (99, 15)):
        a = p * 500.0 ** (-2 * j / 32)
        assert abs(float(t[p, j]) - math.cos(a)) < 2.0 ** -24 and abs(float(t[p, 16 + j]) - math.sin(a)) < 2.0 ** -24
