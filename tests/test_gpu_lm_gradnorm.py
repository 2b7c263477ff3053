"""Norm over many gradients and clipping by it, against 64 bits."""

import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

import paper_1811_10751_b200 as g            # noqa: E402
from lm_reference import check_close           # noqa: E402

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
# FP32 squares: 16 of them are added in a thread before FP64 takes over, each fused step 2^-24; half of that in the root,
# whose result is rounded to FP32
NORM = 9 * 2.0 ** -24


def tensors(sizes, types, scale=1.0, offset=0, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        o = offset[i % len(offset)] if isinstance(offset, (list, tuple)) else offset
        buf = torch.randn(n + o, device="cuda", generator=gen).mul_(scale).to(types[i % len(types)])
        out.append(buf[o:])
    return out


def workspace():
    return torch.full((g.GPD_GRAD_NORM_WORKSPACE // 8,), math.nan, device="cuda", dtype=torch.float64)


def norm_of(grads):
    n = torch.full((1,), math.nan, device="cuda")
    g.gpd_grad_norm(grads, n, workspace())
    return n


def exact_norm(grads):
    return math.sqrt(sum(float(x.double().square().sum()) for x in grads))


SETS = [([1], [F32], 0), ([0, 5, 0], [BF16], 0), ([7, 8, 9, 16, 1, 4096], [F32, BF16, F16], 0), ([8191, 8192, 8193, 40000], [BF16], 0),
        ([100003, 3, 65536, 17], [F32, BF16], [1, 3, 5, 7]), ([20000, 20001], [F16], 1), ([33333] * 5, [F32], [0, 1, 2, 3]),
        ([5000003], [BF16], 5), (list(range(0, 200)), [F32, F16, BF16], [0, 1]), ([300] * 1500, [BF16, F32], 0), ([2000000] * 9, [F16, F32], 0)]


@pytest.mark.parametrize("sizes,types,offset", SETS, ids=[f"{len(s)}x{max(s)}" for s, _, _ in SETS])
def test_norm_and_clipping(sizes, types, offset):
    grads = tensors(sizes, types, 0.1, offset)
    before = [x.clone() for x in grads]
    n, ref = norm_of(grads), exact_norm(grads)
    assert abs(float(n) - ref) <= NORM * ref
    for bound in (ref / 3, ref * 2):
        by = min(1.0, bound / float(n))
        # to other buffers, of another type than the gradient every now and then, which start elsewhere
        out = [torch.full((x.numel() + 4,), 9.0, device="cuda", dtype=[x.dtype, F32, BF16][i % 3]) for i, x in enumerate(grads)]
        views = [o[i % 4:i % 4 + x.numel()] for i, (o, x) in enumerate(zip(out, grads))]
        g.gpd_clip_grads(grads, n, bound, out=views)
        assert all(torch.equal(x, y) for x, y in zip(grads, before))
        for i, (o, v, x) in enumerate(zip(out, views, grads)):
            check_close(v, x.double() * by, 2 * 2.0 ** -24)
            assert bool((o[:i % 4] == 9).all()) and bool((o[i % 4 + x.numel():] == 9).all())
        g.gpd_clip_grads(grads, n, bound)
        for x, y in zip(grads, before):
            check_close(x, y.double() * by, 2 * 2.0 ** -24)
        if bound > ref:
            assert all(torch.equal(x, y) for x, y in zip(grads, before))
        for x, y in zip(grads, before):
            x.copy_(y)


def test_norm_repeats_bit_by_bit():
    grads = tensors([1000003, 77, 500000, 8192], [F32, BF16, F16])
    a = norm_of(grads)
    for _ in range(3):
        assert torch.equal(a, norm_of(grads))


@pytest.mark.parametrize("value", [1e-30, 3e-42, 1e-22, 1e19, 1e35, 3e37])
def test_norms_of_gradients_whose_squares_leave_fp32(value):
    x = torch.full((70001,), value, device="cuda")
    x[::3] = 0
    ref = exact_norm([x])
    if ref > torch.finfo(F32).max:                     # 3e37 * sqrt(46667) = 6.5e39: no FP32 number, rounded to infinity
        assert float(norm_of([x])) == math.inf
        return
    assert abs(float(norm_of([x])) - ref) <= NORM * ref + 2.0 ** -150
    mixed = [x, torch.full((10,), 5.0, device="cuda")]
    ref = exact_norm(mixed)
    assert abs(float(norm_of(mixed)) - ref) <= NORM * ref
    assert float(norm_of([torch.full((4096,), 6e4, device="cuda", dtype=F16)])) == pytest.approx(6e4 * 64, rel=1e-3)


def test_no_gradients_and_zeros():
    assert float(norm_of([])) == 0 and float(norm_of([torch.empty(0, device="cuda")])) == 0
    z = torch.zeros(100000, device="cuda")
    n = norm_of([z])
    assert float(n) == 0
    g.gpd_clip_grads([z], n, 1.0)
    out = [torch.ones_like(z)]
    g.gpd_clip_grads([z], n, 1.0, out=out)
    assert not z.any() and not out[0].any()
    g.gpd_clip_grads([], n, 1.0)


def test_a_norm_that_is_no_number():
    for bad in (math.nan, math.inf, -math.inf):
        x, y = torch.ones(9000, device="cuda"), torch.ones(50, device="cuda", dtype=BF16)
        x[8999] = bad
        n = norm_of([y, x])
        assert math.isnan(float(n)) if math.isnan(bad) else float(n) == math.inf
        g.gpd_clip_grads([y, x], n, 1.0)
        if math.isnan(bad):
            assert torch.isnan(x).all() and torch.isnan(y).all()
        else:
            assert not x[:8999].any() and not y.any() and math.isnan(float(x[8999]))


def test_tensors_of_several_dimensions_in_any_order():
    a = torch.randn((30, 40, 5), device="cuda")
    p = a.permute(2, 0, 1)
    ref = exact_norm([a, a])
    n = norm_of([p, a.clone()])
    assert abs(float(n) - ref) <= NORM * ref
    out = torch.empty_like(a).permute(2, 0, 1)
    g.gpd_clip_grads([p], n, 1.0, out=[out])
    check_close(out, p.double() * (1.0 / float(n)), 2 * 2.0 ** -24)


def test_other_stream_and_graph():
    grads = tensors([100003, 5, 8192 * 40], [F32, BF16])
    out = [torch.zeros_like(x) for x in grads]
    n, ws = torch.empty(1, device="cuda"), workspace()
    st = torch.cuda.Stream()

    def run():
        g.gpd_grad_norm(grads, n, ws, stream=st)
        g.gpd_clip_grads(grads, n, 1.0, out=out, stream=st)
    torch.cuda.synchronize()
    run()
    torch.cuda.synchronize()
    want, wn = [x.clone() for x in out], n.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        run()
    for x in out:
        x.zero_()
    n.zero_()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(n, wn) and all(torch.equal(x, y) for x, y in zip(out, want))


def test_refusals():
    x, y = torch.ones(100, device="cuda"), torch.ones(100, device="cuda", dtype=BF16)
    n, ws = torch.ones(1, device="cuda"), workspace()
    for grads, match in (((x), "list"), ([None], "list"), ([x.double()], "float32"), ([x.cpu()], "cuda"),
                         ([torch.ones((8, 8), device="cuda")[:, :4]], "dense"), ([x[::2]], "dense")):
        with pytest.raises(ValueError, match=match):
            g.gpd_grad_norm(grads, n, ws)
        with pytest.raises(ValueError, match=match):
            g.gpd_clip_grads(grads, n, 1.0)
    with pytest.raises(ValueError):
        g.gpd_grad_norm([x], torch.ones(2, device="cuda"), ws)
    with pytest.raises(ValueError):
        g.gpd_grad_norm([x], n.cpu(), ws)
    with pytest.raises(ValueError):
        g.gpd_grad_norm([x], n, None)
    with pytest.raises(g.GpdError):
        g.gpd_grad_norm([x], n, ws[:-1])
    for bound in (0.0, -1.0, math.nan):
        with pytest.raises(g.GpdError):
            g.gpd_clip_grads([x], n, bound)
    for out in ([], [x, y], [y[:50]], [torch.ones((10, 10), device="cuda")]):
        with pytest.raises(ValueError):
            g.gpd_clip_grads([x], n, 1.0, out=out)
    buf = torch.ones(300, device="cuda")
    for grads, out in (([buf[:100]], [buf[50:150]]), ([x, y], [buf[:100], buf[99:199]]), ([x, x.clone()], [buf[:100], x]),
                       ([x, x], [x, x])):              # the last: clipped twice
        with pytest.raises(g.GpdError):
            g.gpd_clip_grads(grads, n, 1.0, out=out)
    with pytest.raises(g.GpdError):
        g.gpd_clip_grads([x, x], n, 1.0)
    a = torch.ones((4, 6), device="cuda")
    with pytest.raises(ValueError, match="order"):
        g.gpd_clip_grads([a], n, 1.0, out=[torch.ones((6, 4), device="cuda").t()])
    assert bool((x == 1).all()) and bool((buf == 1).all())
