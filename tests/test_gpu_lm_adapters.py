"""Low-rank adapters of many requests beside a shared projection, and their gradients, against the formulas in 64 bits."""

import math
import random

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

import paper_1811_10751_b200 as g            # noqa: E402
from lm_reference import check_close, strided           # noqa: E402

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
# one step of the tensor cores adds 16 products to a sum and truncates: 2^-22 of the terms; chains are 4 to 24 steps long
STEP = 2.0 ** -22


def parts(type, out):
    """What is lost of an FP32 factor that goes through the tensor cores as a sum of 16-bit numbers."""
    return 2.0 ** -22 if type == F16 else 2.0 ** -25 if out == F32 else 2.0 ** -17


def cube(n, rows, cols, dtype, pad, offset):
    buf = torch.empty(offset + n * (rows * (cols + pad) + pad) + 16, dtype=dtype, device="cuda")
    return buf[offset:].as_strided((n, rows, cols), (rows * (cols + pad) + pad, cols + pad, 1))


class Case:
    """lens: rows of the segments; index: their adapters; `before`, `behind`: rows outside of them."""

    def __init__(self, lens, index, n, r, K, N, type=BF16, out=None, grad=F32, pad=0, offset=0, before=0, behind=0, wide=False, seed=0, size=1.0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
        self.n, self.r, self.K, self.N, self.type, self.out_type, self.grad = n, r, K, N, type, out or type, grad
        self.T = T = before + sum(lens) + behind
        cuts = [before]
        for k in lens:
            cuts.append(cuts[-1] + k)
        self.segments = list(zip(cuts[:-1], cuts[1:], index))
        it = torch.int64 if wide else torch.int32
        self.offsets, self.index = torch.tensor(cuts, device="cuda", dtype=it), torch.tensor(index, device="cuda", dtype=it)
        self.pad, self.offset = pad, offset
        self.x, self.dout = self.mat(T, K, type), self.mat(T, N, type)
        self.x.copy_(rand(T, K) * size)
        self.dout.copy_(rand(T, N) * size)
        self.A, self.B = cube(n, r, K, type, pad, offset), cube(n, N, r, type, pad, offset)
        self.A.copy_(rand(n, r, K) / math.sqrt(K))
        self.B.copy_(rand(n, N, r) / math.sqrt(r))
        self.scale = (1.5 + rand(n).abs()).float()
        self.base, self.dbase = self.mat(T, N, self.out_type), self.mat(T, K, self.out_type)
        self.base.copy_(rand(T, N) * size)
        self.dbase.copy_(rand(T, K) * size)

    def mat(self, rows, cols, dtype, fill=None):
        m = strided(rows, cols, dtype, self.pad, self.offset)
        return m if fill is None else m.fill_(fill)

    def forward(self, base="own", scale="own", out=None):
        out = self.mat(self.T, self.N, self.out_type, 77.0) if out is None else out
        h = torch.full((self.T, self.r), 55.0, device="cuda")
        g.gpd_adapter(self.x, self.A, self.B, self.offsets, self.index, out, h, base=self.base if base == "own" else base,
                      scale=self.scale if scale == "own" else scale)
        return out, h

    def check_forward(self, out, h, base="own", scaled=True):
        covered = torch.zeros(self.T, dtype=torch.bool, device="cuda")
        for a, b, i in self.segments:
            covered[a:b] = True
            own = self.base[a:b].double() if isinstance(base, str) else 0 * out[a:b].double() if base is None else base[a:b].double()
            if i < 0:
                assert not h[a:b].any()
                assert torch.equal(out[a:b].double(), own)
                continue
            if i >= self.n:
                assert torch.isnan(h[a:b]).all() and torch.isnan(out[a:b]).all()
                continue
            x, A, B = self.x[a:b].double(), self.A[i].double(), self.B[i].double()
            check_close(h[a:b], x @ A.t(), 4 * STEP + (self.K / 64 + 16) * 2.0 ** -24, x.abs() @ A.abs().t())
            s = float(self.scale[i]) if scaled else 1.0
            hd = h[a:b].double()
            hs = hd.abs().amax(1, keepdim=True).expand_as(hd) if self.type == F16 else hd.abs()
            check_close(out[a:b], own + s * (hd @ B.t()), parts(self.type, self.out_type) + 26 * STEP, own.abs() + s * (hs @ B.abs().t()))
        assert bool((out[~covered] == 77).all()) and bool((h[~covered] == 55).all())

    def workspace(self):
        n = g.gpd_adapter_backward_workspace(self.T, self.K, self.N, self.n, self.r)
        return torch.full((n,), 255, dtype=torch.uint8, device="cuda")         # NaN wherever it is read unwritten

    def backward(self, h, **kw):
        self.dx = kw.pop("dx", None)
        if self.dx is None:
            self.dx = self.mat(self.T, self.K, self.out_type, 77.0)
        self.dA, self.dB = (cube(self.n, *s, self.grad, self.pad, self.offset).fill_(3.0) for s in ((self.r, self.K), (self.N, self.r)))
        args = dict(dbase=self.dbase, scale=self.scale) | kw
        g.gpd_adapter_backward(self.dout, self.x, self.A, self.B, h, self.offsets, self.index, self.dx, self.dA, self.dB, self.workspace(), **args)

    def check_backward(self, h, accumulate=False):
        dA, dB, sA, sB, mA, mB = (torch.zeros(s, device="cuda", dtype=torch.float64) for s in 3 * [(self.n, self.r, self.K), (self.n, self.N, self.r)])
        covered = torch.zeros(self.T, dtype=torch.bool, device="cuda")
        lost_u = 4 * STEP + (self.N / 64 + 16) * 2.0 ** -24
        for a, b, i in self.segments:
            covered[a:b] = True
            if i < 0:
                assert torch.equal(self.dx[a:b], self.dbase[a:b])
                continue
            if i >= self.n:
                assert torch.isnan(self.dx[a:b]).all()
                continue
            d, x, A, B, hd, s = self.dout[a:b].double(), self.x[a:b].double(), self.A[i].double(), self.B[i].double(), h[a:b].double(), float(self.scale[i])
            u, us = s * (d @ B), s * (d.abs() @ B.abs())
            um = us.amax(1, keepdim=True).expand_as(us) if self.type == F16 else us
            own = self.dbase[a:b].double()
            check_close(self.dx[a:b], own + u @ A, lost_u + parts(self.type, self.out_type) + 26 * STEP, own.abs() + um @ A.abs())
            if a == b:
                continue
            top = (lambda v: v.amax(0, keepdim=True).expand_as(v)) if self.type == F16 else (lambda v: v)
            dA[i] += u.t() @ x
            sA[i] += top(us).t() @ x.abs()
            dB[i] += s * (d.t() @ hd)
            sB[i] += s * (d.abs().t() @ top(hd.abs()))
        lost = parts(self.type, self.grad) + 14 * STEP + (self.T / 64 + 40) * 2.0 ** -24
        old = 3.0 if accumulate else 0.0
        check_close(self.dA, dA + old, lost + lost_u, sA + old)
        check_close(self.dB, dB + old, lost, sB + old)
        if not accumulate and self.grad == F32:        # as a whole: FP32's own rounding, and little more
            for got, ref in ((self.dA, dA), (self.dB, dB)):
                assert float((got.double() - ref).norm()) <= 2e-6 * float(ref.norm())
        assert bool((self.dx[~covered] == 77).all())


def ragged(T, S, n, seed, without=False):
    rng = random.Random(seed)
    cuts = sorted(rng.randint(0, T) for _ in range(S - 1))
    index = [rng.randrange(-1 if without else 0, n) for _ in range(S)]
    return dict(lens=[b - a for a, b in zip([0] + cuts, cuts + [T])], index=index, n=n)


CASES = {
    "one row": dict(lens=[1], index=[0], n=1, r=16, K=256, N=256),
    "one row each": dict(lens=[1] * 37, index=[(7 * i) % 40 for i in range(37)], n=40, r=16, K=1024, N=512),
    "one row each f16, adapters shared": dict(lens=[1] * 20, index=[i % 3 for i in range(20)], n=3, r=8, K=512, N=1000, type=F16),
    "one row each, many, wide factors": dict(**ragged(300, 290, 17, 20, True), r=32, K=1416, N=2000),
    "one row each, too wide to be held": dict(lens=[1, 2, 1], index=[2, 0, 1], n=3, r=128, K=8192, N=4096),
    "few rows each f32 out": dict(**ragged(90, 13, 5, 21), r=64, K=200, N=72, out=F32, before=3, behind=4),
    "few rows each rank 128": dict(**ragged(60, 9, 5, 22), r=128, K=512, N=576, type=F16),
    "short": dict(lens=[3, 0, 16, 17, 1, 40, 2], index=[1, 0, -1, 2, 2, 0, 1], n=3, r=32, K=320, N=704, wide=True),
    "ragged": dict(**ragged(700, 5, 3, 1, True), r=64, K=512, N=768),
    "ragged f16, f32 out": dict(**ragged(515, 4, 2, 2), r=16, K=640, N=256, type=F16, out=F32),
    "f32 out": dict(**ragged(300, 3, 2, 3), r=128, K=320, N=448, out=F32),
    "rank 1": dict(**ragged(130, 3, 2, 4), r=1, K=64, N=72),
    "rank 7, odd": dict(**ragged(200, 6, 4, 5), r=7, K=333, N=251),
    "rank 65": dict(**ragged(150, 3, 2, 6), r=65, K=136, N=136, type=F16),
    "rank 4, adapters without rows": dict(lens=[70, 80], index=[5, 2], n=7, r=4, K=96, N=200, grad=BF16),
    "rows outside": dict(lens=[30, 5], index=[0, 1], n=2, r=16, K=128, N=128, before=9, behind=70),
    "no such adapter": dict(lens=[20, 30, 4], index=[0, 9, 1], n=2, r=16, K=128, N=200),
    "strides": dict(**ragged(200, 4, 2, 7), r=24, K=200, N=264, pad=8),
    "rows off boundaries": dict(**ragged(200, 4, 2, 8), r=24, K=200, N=264, pad=3, offset=1),
    "off boundaries f32 out": dict(**ragged(70, 2, 2, 9), r=16, K=100, N=131, pad=1, offset=1, out=F32, type=F16),
    "one adapter, many rows": dict(lens=[5000], index=[0], n=1, r=16, K=512, N=384),
    "many rows, several runs": dict(lens=[1500, 700, 900, 2100], index=[1, 0, 1, 2], n=3, r=40, K=264, N=136, grad=BF16),
    "many segments": dict(**ragged(900, 300, 11, 10, True), r=16, K=128, N=128),
    "several runs f16": dict(lens=[900, 1300], index=[0, 1], n=2, r=16, K=128, N=256, type=F16, grad=F16),
    "several runs each, ends in tiles": dict(lens=[700, 1, 1290, 0, 333, 65], index=[1, 0, 1, 0, 0, 1], n=2, r=64, K=520, N=1160, grad=F32),
    "rank 128, runs": dict(lens=[650, 1001], index=[0, 1], n=2, r=128, K=256, N=136, type=F16),
    "long sums": dict(lens=[60], index=[0], n=1, r=16, K=20000, N=16),
    "wide": dict(lens=[50], index=[0], n=1, r=16, K=16, N=20000),
    "tiny f16": dict(**ragged(150, 3, 2, 11), r=16, K=128, N=128, type=F16, size=2e-6),
    "large f16": dict(**ragged(150, 3, 2, 12), r=16, K=128, N=128, type=F16, size=2e3, out=F32),
}


@pytest.mark.parametrize("name", CASES)
def test_forward_and_gradients(name):
    c = Case(**CASES[name])
    out, h = c.forward()
    c.check_forward(out, h)
    hb = torch.where(torch.isfinite(h), h, 0.0)
    c.backward(hb)
    c.check_backward(hb)
    assert g.gpd_device_status() == 0


def test_base_in_place_left_out_and_no_scale():
    c = Case(**CASES["ragged"])
    out, h = c.forward()
    base = c.base.clone()
    same, h2 = c.forward(out=c.base)
    covered = slice(0, c.T)
    assert torch.equal(same[covered], out[covered]) and torch.equal(h, h2)
    c.base.copy_(base)
    out, h = c.forward(base=None)
    c.check_forward(out, h, base=None)
    out, h = c.forward(scale=None)
    c.check_forward(out, h, scaled=False)
    c.scale.fill_(1.0)
    c.backward(h, dx=c.dbase.clone())
    dx, dA, dB = c.dx, c.dA, c.dB
    c.backward(h, scale=None)
    assert torch.equal(c.dA, dA) and torch.equal(c.dB, dB) and torch.equal(c.dx, dx)
    in_place = c.dbase
    c.backward(h, dx=in_place)
    assert torch.equal(in_place, dx)


def test_accumulation_and_parts_left_out():
    c = Case(**CASES["many rows, several runs"])
    _, h = c.forward()
    c.backward(h, accumulate=True)
    c.check_backward(h, accumulate=True)
    c.backward(h)
    dA, dB, dx, ws = c.dA, c.dB, c.dx, c.workspace()
    args = (c.dout, c.x, c.A, c.B, h, c.offsets, c.index)
    dA2, dB2, dx2 = torch.zeros_like(dA), torch.zeros_like(dB), torch.zeros_like(dx)
    g.gpd_adapter_backward(*args, None, dA2, dB2, ws, scale=c.scale)
    g.gpd_adapter_backward(*args, dx2, None, None, ws, dbase=c.dbase, scale=c.scale)
    assert torch.equal(dA, dA2) and torch.equal(dB, dB2) and torch.equal(dx, dx2)
    c.backward(h)
    assert torch.equal(dA, c.dA) and torch.equal(dB, c.dB)             # bit by bit


def test_no_rows_no_segments_no_adapters():
    c = Case(lens=[10], index=[0], n=2, r=8, K=64, N=64)
    ws = c.workspace()
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    h = torch.full((10, 8), 5.0, device="cuda")
    out = torch.full((10, 64), 7.0, device="cuda", dtype=BF16)
    g.gpd_adapter(c.x, c.A, c.B, c.offsets[:1], none, out, h)
    g.gpd_adapter(c.x[:0], c.A, c.B, torch.zeros(2, dtype=torch.int32, device="cuda"), c.index, out[:0], h[:0])
    assert bool((out == 7).all()) and bool((h == 5).all())
    dA, dB = torch.ones((2, 8, 64), device="cuda"), torch.ones((2, 64, 8), device="cuda")
    g.gpd_adapter_backward(c.dout, c.x, c.A, c.B, h, c.offsets[:1], none, out, dA, dB, ws)
    assert not dA.any() and not dB.any() and bool((out == 7).all())
    g.gpd_adapter(c.x, c.A[:0], c.B[:0], c.offsets, torch.full((1,), -1, dtype=torch.int32, device="cuda"), out, h, base=c.base)
    assert torch.equal(out, c.base) and not h.any()


def test_offsets_outside_the_batch_stay_inside_it():
    """Bad offsets have no meaning, but nothing beyond the tensors is touched."""
    c = Case(lens=[40, 40], index=[0, 1], n=2, r=16, K=64, N=64)
    for bad in ([-5, 40, 1000], [60, 20, 70], [90, 95, 99], [0, 80, 40]):
        o = torch.tensor(bad, dtype=torch.int32, device="cuda")
        h, out = torch.zeros((80, 16), device="cuda"), torch.zeros((81, 64), device="cuda", dtype=BF16)
        g.gpd_adapter(c.x, c.A, c.B, o, c.index, out[:80], h, base=c.base)
        dA, dB = torch.zeros((2, 16, 64), device="cuda"), torch.zeros((2, 64, 16), device="cuda")
        g.gpd_adapter_backward(c.dout, c.x, c.A, c.B, h, o, c.index, out[:80], dA, dB, c.workspace())
        torch.cuda.synchronize()
        assert not out[80].any() and torch.isfinite(out).all()


def test_infinities_and_nans_stay_in_their_rows():
    for type in (BF16, F16):
        c = Case(lens=[30, 20], index=[0, 1], n=2, r=16, K=128, N=96, type=type)
        clean, _ = c.forward()
        c.x[3, 5], c.x[40, 7], c.x[41, 0] = math.nan, math.inf, -math.inf
        out, h = c.forward()
        bad = torch.zeros(50, dtype=torch.bool, device="cuda")
        bad[[3, 40, 41]] = True
        assert torch.equal(~torch.isfinite(h).any(1), bad) and torch.equal(out[~bad], clean[~bad])
        assert torch.isnan(out[3]).all() and not torch.isfinite(out[40:42]).any()


@pytest.mark.parametrize("type", [BF16, F16])
@pytest.mark.parametrize("lens", [[70, 90, 61], [5, 9, 3]])
def test_gradients_of_an_adapter_do_not_see_the_rows_of_others(type, lens):
    c = Case(lens=lens, index=[0, 1, 2], n=3, r=16, K=128, N=192, type=type)
    _, h = c.forward()
    c.backward(h)
    dx, dA, dB = c.dx.clone(), c.dA.clone(), c.dB.clone()
    a, b = lens[0], lens[0] + lens[1]
    c.x[a, 3], c.x[b - 1, 100], c.dout[a, 5], c.dout[b - 1, 191], h[a, 2], h[b - 1, 7] = math.nan, math.inf, -math.inf, math.nan, math.nan, math.inf
    c.backward(h)
    others = torch.ones(c.T, dtype=torch.bool, device="cuda")
    others[a:b] = False
    assert torch.equal(c.dx[others], dx[others])
    for i in (0, 2):
        assert torch.equal(c.dA[i], dA[i]) and torch.equal(c.dB[i], dB[i])
    assert not torch.isfinite(c.dA[1]).all() and not torch.isfinite(c.dB[1]).all()


def test_gradients_agree_with_differences():
    c = Case(lens=[5, 4], index=[1, 0], n=2, r=3, K=6, N=7, out=F32)
    _, h = c.forward()
    c.backward(h)

    def loss(x, A, B):
        return sum(float(((float(c.scale[i]) * (x[a:b] @ A[i].t()) @ B[i].t()) * c.dout[a:b].double()).sum()) for a, b, i in c.segments)
    args = [c.x.double(), c.A.double(), c.B.double()]
    got = [c.dx.double() - c.dbase.double(), c.dA.double(), c.dB.double()]
    step = 2.0 ** -12                                  # the loss is linear in each argument: differences are exact but for rounding
    for which, places in ((0, [(0, 0), (8, 5), (4, 3)]), (1, [(0, 0, 0), (1, 2, 5)]), (2, [(0, 6, 2), (1, 3, 1)])):
        for at in places:
            up, down = [v.clone() for v in args], [v.clone() for v in args]
            up[which][at] += step
            down[which][at] -= step
            d = (loss(*up) - loss(*down)) / (2 * step)
            # dB takes h, dA and dx take u as FP32 sums of at most 7 terms of order one each
            assert abs(d - float(got[which][at])) < 1e-4


def test_other_stream_and_graph():
    c = Case(**CASES["many rows, several runs"])
    out, h = c.mat(c.T, c.N, BF16, 0.0), torch.zeros((c.T, c.r), device="cuda")
    dx, dA, dB, ws = torch.zeros_like(c.x), torch.zeros(c.A.shape, device="cuda"), torch.zeros(c.B.shape, device="cuda"), c.workspace()
    st = torch.cuda.Stream()

    def run():
        g.gpd_adapter(c.x, c.A, c.B, c.offsets, c.index, out, h, base=c.base, scale=c.scale, stream=st)
        g.gpd_adapter_backward(c.dout, c.x, c.A, c.B, h, c.offsets, c.index, dx, dA, dB, ws, dbase=c.dbase, scale=c.scale, stream=st)
    torch.cuda.synchronize()
    run()
    torch.cuda.synchronize()
    results = (out, h, dx, dA, dB)
    want = [t.clone() for t in results]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        run()
    for t in results:
        t.zero_()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(results, want))


@pytest.mark.parametrize("type", [BF16, F16])
@pytest.mark.parametrize("r", [32, 64, 128])
def test_long_sums_while_their_stages_are_filled_again(r, type):
    """16384 rows of 8192 columns, so that the copies run ahead of the products all the time: every row is right, in every run."""
    c = Case([700] * 23 + [284], [i % 4 for i in range(24)], 4, r, 8192, 256, type, seed=r)
    out, h = c.forward()
    c.check_forward(out, h)
    for _ in range(12):
        again = c.forward(out=c.mat(c.T, c.N, c.out_type, 77.0))
        assert torch.equal(again[1], h) and torch.equal(again[0], out)


def test_what_follows_a_batch_without_adapters_sees_its_zeros():
    """In place and without adapters the second product has nothing to do; the next call still comes after the first one."""
    T, r, K, N = 300000, 128, 8, 64
    x, out = torch.ones(T, K, dtype=BF16, device="cuda"), torch.ones(T, N, dtype=BF16, device="cuda")
    A, B = torch.ones(1, r, K, dtype=BF16, device="cuda"), torch.ones(1, N, r, dtype=BF16, device="cuda")
    offsets, index = torch.tensor([0, T // 3, T], device="cuda"), torch.tensor([-1, -1], device="cuda")
    h = torch.empty(T, r, device="cuda")
    norm, ws = torch.empty(1, device="cuda"), torch.empty(g.GPD_GRAD_NORM_WORKSPACE, dtype=torch.uint8, device="cuda")
    for _ in range(5):
        h.fill_(55)
        g.gpd_adapter(x, A, B, offsets, index, out, h, base=out)
        g.gpd_grad_norm([h], norm, ws)
        assert float(norm) == 0
        assert not h.any() and bool((out == 1).all())


def test_refusals():
    c = Case(lens=[10, 6], index=[0, 1], n=2, r=8, K=64, N=48)
    h, out = torch.zeros((16, 8), device="cuda"), torch.zeros((16, 48), device="cuda", dtype=BF16)
    ok = dict(x=c.x, A=c.A, B=c.B, offsets=c.offsets, index=c.index, out=out, h=h, base=c.base, scale=c.scale)
    g.gpd_adapter(**ok)

    def refused(match, **kw):
        with pytest.raises(ValueError, match=match):
            g.gpd_adapter(**{**ok, **kw})
    refused("bfloat16", x=c.x.float())
    refused("bfloat16", A=c.A.half())
    refused("bfloat16", B=c.B.half())
    refused("A", A=c.A[0])
    refused("A", A=c.A[:, :, :60])
    refused("B", B=c.B[:1])
    refused("B", B=c.B[:, :, :7])
    refused("A", A=torch.zeros((2, 129, 64), device="cuda", dtype=BF16), B=torch.zeros((2, 48, 129), device="cuda", dtype=BF16))
    refused("offsets", offsets=c.offsets[:2])
    refused("one type", offsets=c.offsets.long())
    refused("index", index=c.index.float())
    refused("out", out=out[:, :40])
    refused("out", out=out.half())
    refused("base", base=c.base.float())
    refused("h", h=h[:, :4])
    refused("h", h=None)
    refused("scale", scale=c.scale[:1])
    refused("cuda", index=c.index.cpu())
    dA, dB, dx = torch.zeros((2, 8, 64), device="cuda"), torch.zeros((2, 48, 8), device="cuda"), torch.zeros_like(c.x)
    back = dict(dout=c.dout, x=c.x, A=c.A, B=c.B, h=h, offsets=c.offsets, index=c.index, dx=dx, dA=dA, dB=dB, workspace=c.workspace())
    g.gpd_adapter_backward(**back)
    for kw in (dict(dA=None), dict(dB=dB.bfloat16()), dict(dx=None, dbase=dx), dict(dout=c.dout.float()), dict(workspace=None), dict(dA=dA[:, :, :63])):
        with pytest.raises(ValueError):
            g.gpd_adapter_backward(**{**back, **kw})
    with pytest.raises(g.GpdError):
        g.gpd_adapter_backward(**{**back, "workspace": back["workspace"][:-1]})
    with pytest.raises(g.GpdError):
        g.gpd_adapter_backward_workspace(10, 64, 48, 2, 129)
