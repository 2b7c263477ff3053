"""8-bit product with block scales against the 64-bit product of the numbers that the operands stand for.

Integer operands with small scale exponents make every partial sum an integer multiple of one power of two
below 2^24 of it: the FP32 result has to be exact whatever the order.  For random operands the bound is the
sum of magnitudes times 2^-23 (one truncation) for each instruction of 32 terms in a chain and for each
addition of a chain, plus four for the alignment inside the instructions: 16-bit results have one chain of K / 32,
FP32 results chains of at
most 32, held to the bound of chains of 16 with K / 512 additions."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

import paper_1811_10751_b200 as g                                           # noqa: E402
from tests.lm_reference import check_close, scale_values, spread, strided   # noqa: E402

E4, E5 = torch.float8_e4m3fn, torch.float8_e5m2
BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32

SHAPES = [(1, 1, 1), (1, 16, 16), (1, 128, 128), (7, 4096, 4096), (16, 4096, 1000), (17, 200, 300), (33, 136, 5000),
          (64, 1000, 4100), (128, 128, 128), (129, 257, 385), (200, 8192, 640), (300, 4096, 1024), (512, 8192, 1024),
          (1000, 1000, 1000), (130, 130, 8192), (2048, 2048, 512), (4096, 4100, 300), (3, 50000, 256), (5000, 24, 160)]


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _operand(seed, rows, cols, dtype, block_rows, integers):
    """8-bit matrix with scales, in padded buffers full of NaN."""
    q, s = g.new_fp8(rows, cols, dtype, block_rows)
    q._base.view(torch.uint8).fill_(0x7F)
    s._base.view(torch.uint8).fill_(0xFF)
    if integers:
        q.copy_(torch.randint(-4, 5, (rows, cols), device="cuda", generator=_gen(seed)).float())
        s.view(torch.uint8).copy_(torch.randint(126, 129, s.shape, device="cuda", generator=_gen(seed + 1)))
    else:
        top = 3.0 if dtype == E4 else 100.0
        q.copy_(torch.randn((rows, cols), device="cuda", generator=_gen(seed)) * top)
        s.view(torch.uint8).copy_(torch.randint(117, 133, s.shape, device="cuda", generator=_gen(seed + 1)))
    return q, s, q.double() * spread(scale_values(s), block_rows, rows, cols)


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("at,bt,ar,br,out", [(E4, E4, 1, 128, F32), (E5, E4, 1, 1, F32), (E4, E5, 128, 1, BF), (E5, E5, 1, 128, HF)])
def test_integer_operands_are_exact(M, N, K, at, bt, ar, br, out):
    A, sa, a = _operand(1, M, K, at, ar, True)
    B, sb, b = _operand(5, N, K, bt, br, True)
    D = strided(M, N, out, pad=5)
    D.fill_(float("nan"))
    g.gpd_gemm_fp8(A, sa, B, sb, D)
    assert g.gpd_device_status() == 0
    ref = a @ b.t()
    assert torch.equal(D, ref.to(out) if out != F32 else ref.float())
    prev = torch.randint(-8, 9, (M, N), device="cuda", generator=_gen(9)).to(out)
    D.copy_(prev)
    g.gpd_gemm_fp8(A, sa, B, sb, D, accumulate=True)
    assert torch.equal(D, (ref + prev.double()).to(out))


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("at,bt,ar,br,out", [(E4, E4, 1, 128, BF), (E5, E4, 1, 1, F32), (E4, E4, 1, 128, F32)])
def test_random_operands_within_the_bound(M, N, K, at, bt, ar, br, out):
    A, sa, a = _operand(1, M, K, at, ar, False)
    B, sb, b = _operand(5, N, K, bt, br, False)
    D = torch.empty((M, N), dtype=out, device="cuda")
    g.gpd_gemm_fp8(A, sa, B, sb, D)
    assert g.gpd_device_status() == 0
    n = (20 + K / 512) if out == F32 else (K / 32 + 4)
    check_close(D, a @ b.t(), 0.0 if n == 0 else n * 2.0 ** -23, a.abs() @ b.abs().t())
    D2 = torch.empty_like(D)
    for _ in range(3):                                                      # no order that changes
        g.gpd_gemm_fp8(A, sa, B, sb, D2)
        assert torch.equal(D, D2)


def test_layer_forward_and_both_gradients_from_one_cut():
    """X W^T, Delta W and Delta^T X from straight and transposed cuts, against the products of what the cuts hold."""
    T, N, K = 200, 384, 520
    X, W, D = (torch.randn(s, device="cuda", generator=_gen(i)) for i, s in enumerate(((T, K), (N, K), (T, N))))

    def cut(x, dtype, br):
        r, c = x.shape
        q, s = g.new_fp8(r, c, dtype, br)
        qT, sT = g.new_fp8(c, r, dtype, br)
        g.gpd_quantize_blocks(x, q=q, scales=s, qT=qT, scalesT=sT, block_rows=br)
        val = lambda q, s: q.double() * spread(scale_values(s), br, *q.shape)   # noqa: E731
        return q, s, val(q, s), qT, sT, val(qT, sT)
    xq, xs, xv, xqT, xsT, xvT = cut(X, E4, 1)
    wq, ws, wv, wqT, wsT, wvT = cut(W, E4, 128)
    dq, ds, dv, dqT, dsT, dvT = cut(D, E5, 1)
    assert torch.equal(wvT, wv.t())
    for args, ref, size in (((xq, xs, wq, ws), xv @ wv.t(), xv.abs() @ wv.abs().t()),
                            ((dq, ds, wqT, wsT), dv @ wv, dv.abs() @ wv.abs()),
                            ((dqT, dsT, xqT, xsT), dvT @ xvT.t(), dvT.abs() @ xvT.abs().t())):
        out = torch.empty(ref.shape, device="cuda")
        g.gpd_gemm_fp8(*args, out)
        check_close(out, ref, 22 * 2.0 ** -23, size)


def test_nan_scale_shows_and_stays_in_its_row():
    A, sa, a = _operand(1, 130, 256, E4, 1, True)
    B, sb, b = _operand(5, 140, 256, E4, 1, True)
    sa[3].view(torch.uint8)[1] = 255
    out = torch.empty((130, 140), device="cuda")
    g.gpd_gemm_fp8(A, sa, B, sb, out)
    assert bool(torch.isnan(out[3]).all())
    keep = torch.arange(130, device="cuda") != 3
    assert torch.equal(out[keep], (a @ b.t())[keep].float())


def test_empty_products_and_refusals():
    e = torch.empty((0, 16), device="cuda", dtype=E4)
    A, sa, _ = _operand(1, 4, 160, E4, 1, True)
    g.gpd_gemm_fp8(A, sa, g.new_fp8(0, 160)[0], g.new_fp8(0, 160)[1], torch.empty((4, 0), device="cuda"))
    q0, s0 = g.new_fp8(4, 0)
    out = torch.full((4, 4), 3.0, device="cuda")
    g.gpd_gemm_fp8(q0, s0, q0, s0, out, accumulate=True)
    assert bool((out == 3).all())
    g.gpd_gemm_fp8(q0, s0, q0, s0, out)
    assert bool((out == 0).all())
    B, sb, _ = _operand(1, 4, 160, E4, 1, True)
    for args in ((A.float(), sa, B, sb, out), (A, sa[:2], B, sb, out), (A, sa, B[:, :128], sb, out), (A, sa, B, sb, out[:3]),
                 (A, sa[:, :1], B, sb, out), (A.cpu(), sa.cpu(), B, sb, out), (A, sa, B, sb, out.t().double()), (A, sa.float(), B, sb, out)):
        with pytest.raises(ValueError):
            g.gpd_gemm_fp8(*args)
    tight = torch.zeros((4, 161), device="cuda", dtype=torch.uint8).view(E4)           # rows at odd bytes
    with pytest.raises(g.GpdError) as err:
        g.gpd_gemm_fp8(tight, g.new_fp8(4, 161)[1], tight, g.new_fp8(4, 161)[1], out)
    assert err.value.status == g.GPD_ERR_ARG
    p = A.data_ptr()
    call = g.lib.gpd_gemm_fp8
    assert call(0, p, 160, p, 4, 1, 3, p, 160, p, 4, 1, 0, p, 4, 4, 4, 160, 0, None) == g.GPD_ERR_ARG
    assert call(3, p, 160, p, 4, 2, 3, p, 160, p, 4, 1, 0, p, 4, 4, 4, 160, 0, None) == g.GPD_ERR_ARG
    assert call(3, p, 144, p, 4, 1, 3, p, 160, p, 4, 1, 0, p, 4, 4, 4, 160, 0, None) == g.GPD_ERR_SHAPE
    assert call(3, p, 160, p, 1, 1, 3, p, 160, p, 4, 1, 0, p, 4, 4, 4, 160, 0, None) == g.GPD_ERR_SHAPE
    assert call(3, p, 160, p, 4, 1, 3, p, 160, p, 4, 1, 0, p, 3, 4, 4, 160, 0, None) == g.GPD_ERR_SHAPE
    assert call(3, p, 160, None, 4, 1, 3, p, 160, p, 4, 1, 0, p, 4, 4, 4, 160, 0, None) == g.GPD_ERR_ARG
    del e
