"""Norms of queries and keys per head with rotation by position, and their gradient, against the formulas in 64 bits."""

import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

import paper_1811_10751_b200 as g            # noqa: E402
from lm_reference import check_close, strided           # noqa: E402

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
EPS = 1e-6
# FP32 steps behind a result: at most 8 additions in a thread, 5 over lanes, one division, the root (2 units), three
# products and one fused step, each 2^-24 of its operands
STEPS = 20 * 2.0 ** -24


def turn(x, table, pos, axes, neighbours, back=False):
    """x [T, H, D] in 64 bits, pairs turned by table[pos]; and the sizes of the terms that every result is made of."""
    half = table.shape[1] // 2
    y, size = x.clone(), x.abs().clone()
    for j in range(half):
        p = pos if pos.dim() == 1 else pos[:, int(axes[j])]
        row = table.double()[p.long()]
        c, s = row[:, j, None], row[:, half + j, None] * (-1 if back else 1)
        i, k = (2 * j, 2 * j + 1) if neighbours else (j, j + half)
        a, b = x[:, :, i], x[:, :, k]
        y[:, :, i], y[:, :, k] = a * c - b * s, b * c + a * s
        size[:, :, i] = size[:, :, k] = a.abs() + b.abs()
    return y, size


def forward(x, w, table, pos, axes, neighbours):
    z = x.double()
    if w is not None:
        z = z / torch.sqrt(z.square().mean(2, keepdim=True) + EPS) * w.double()
    return turn(z, table, pos, axes, neighbours) if table is not None else (z, z.abs())


def backward(dy, x, w, table, pos, axes, neighbours):
    gr, size = dy.double(), dy.double().abs()
    if table is not None:
        gr, size = turn(gr, table, pos, axes, neighbours, back=True)
    if w is None:
        return gr, size, None, None
    x = x.double()
    s = 1 / torch.sqrt(x.square().mean(2, keepdim=True) + EPS)
    gw, sw = gr * w.double(), size * w.double().abs()
    dx = s * (gw - x * s * s * (gw * x).mean(2, keepdim=True))
    dsize = s * (sw + x.abs() * s * s * (sw * x.abs()).mean(2, keepdim=True))
    return dx, dsize, (gr * x * s).sum((0, 1)), (size * x.abs() * s).sum((0, 1))


class Case:
    def __init__(self, T, Hq, Hk, D, R, type=BF16, axes=1, neighbours=False, norm=True, wtype=None, pad=0, offset=0, P=97, index=torch.int32,
                 seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
        self.T, self.Hq, self.Hk, self.D, self.norm, self.neighbours = T, Hq, Hk, D, norm, neighbours
        self.fused = strided(T, (Hq + 2 * Hk) * D, type, pad, offset)
        self.fused.copy_(rand(T, (Hq + 2 * Hk) * D) * 3)
        self.q, self.k = self.fused[:, :Hq * D], self.fused[:, Hq * D:(Hq + Hk) * D]
        self.wq, self.wk = [(1 + 0.3 * rand(D)).to(wtype or type) for _ in range(2)] if norm else (None, None)
        self.table = g.new_rope_table(P, R) if R else None
        self.axes = torch.randint(0, axes, (R // 2,), device="cuda", generator=gen, dtype=torch.uint8) if axes > 1 else None
        self.pos = torch.randint(0, P, (T, axes) if axes > 1 else (T,), device="cuda", generator=gen, dtype=index) if R else None
        self.dq, self.dk = (strided(T, h * D, type, pad, offset) for h in (Hq, Hk))
        self.dq.copy_(rand(T, Hq * D))
        self.dk.copy_(rand(T, Hk * D))
        self.pad, self.offset, self.type = pad, offset, type

    def out(self, H):
        o = strided(self.T, H * self.D, self.type, self.pad, self.offset)
        o.fill_(7.0)
        return o

    def args(self):
        return dict(q_weight=self.wq, k_weight=self.wk, eps=EPS, axes=self.axes, neighbours=self.neighbours)

    def heads(self, x):
        return x.reshape(self.T, -1, self.D)

    def check_forward(self, qo, ko):
        for x, w, o in ((self.q, self.wq, qo), (self.k, self.wk, ko)):
            ref, size = forward(self.heads(x), w, self.table, self.pos, self.axes, self.neighbours)
            check_close(o, ref.flatten(1), STEPS, size.flatten(1))

    def backward(self, dqi, dki, **kw):
        self.dw = [torch.full((self.D,), math.nan, device="cuda") for _ in range(2)] if self.norm else [None, None]
        ws = torch.full((2 * g.GPD_HEAD_NORM_MAX_PARTS * self.D,), math.nan, device="cuda") if self.norm else None
        g.gpd_head_norm_rope_backward(self.dq, self.dk, self.q, self.k, self.table, self.pos, dqi, dki, self.D, dq_weight=self.dw[0],
                                      dk_weight=self.dw[1], workspace=ws, **self.args(), **kw)

    def check_backward(self, dqi, dki, dq=None, dk=None):
        for x, dy, w, o, dw in ((self.q, self.dq if dq is None else dq, self.wq, dqi, self.dw[0]),
                                (self.k, self.dk if dk is None else dk, self.wk, dki, self.dw[1])):
            ref, size, wref, wsize = backward(self.heads(dy), self.heads(x), w, self.table, self.pos, self.axes, self.neighbours)
            check_close(o, ref.flatten(1), 2 * STEPS, size.flatten(1))
            if self.norm:                              # one addition per token and head at most, beside the steps above
                check_close(dw, wref, 2 * STEPS + self.T * x.shape[1] // self.D * 2.0 ** -24, wsize)


CASES = [dict(T=1, Hq=1, Hk=1, D=128, R=128), dict(T=8, Hq=32, Hk=8, D=128, R=128), dict(T=5, Hq=5, Hk=1, D=64, R=32, type=F16),
         dict(T=300, Hq=9, Hk=3, D=80, R=80, neighbours=True), dict(T=1100, Hq=16, Hk=2, D=128, R=64, neighbours=True, type=F16),
         dict(T=33, Hq=7, Hk=7, D=112, R=112, axes=3), dict(T=200, Hq=4, Hk=4, D=256, R=256, axes=4, neighbours=True, index=torch.int64),
         dict(T=61, Hq=3, Hk=1, D=128, R=128, type=F32), dict(T=40, Hq=2, Hk=1, D=96, R=24, type=F32, neighbours=True),
         dict(T=19, Hq=4, Hk=2, D=2, R=2), dict(T=21, Hq=3, Hk=2, D=6, R=4, type=F32), dict(T=50, Hq=3, Hk=2, D=254, R=254, type=F16),
         dict(T=37, Hq=3, Hk=2, D=130, R=62, neighbours=True), dict(T=44, Hq=4, Hk=2, D=72, R=40, wtype=F32),
         dict(T=29, Hq=4, Hk=2, D=128, R=128, pad=1), dict(T=29, Hq=4, Hk=2, D=128, R=128, pad=4, offset=4),
         dict(T=31, Hq=4, Hk=2, D=128, R=128, offset=3, axes=2, index=torch.int64), dict(T=31, Hq=4, Hk=2, D=64, R=64, type=F32, pad=2),
         dict(T=70, Hq=6, Hk=2, D=128, R=0), dict(T=77, Hq=13, Hk=5, D=80, R=40, type=F32),
         dict(T=130, Hq=7, Hk=3, D=96, R=96, wtype=F32), dict(T=600, Hq=12, Hk=12, D=48, R=48), dict(T=3, Hq=2, Hk=64, D=64, R=64, wtype=F32, type=F16),
         dict(T=65, Hq=8, Hk=8, D=80, R=80, norm=False, axes=3, neighbours=True, type=F16), dict(T=9, Hq=4, Hk=2, D=128, R=96, norm=False),
         dict(T=12, Hq=3, Hk=1, D=10, R=6, norm=False, type=F32)]
IDS = ["-".join(f"{k}{str(v).replace('torch.', '')}" for k, v in c.items()) for c in CASES]


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_forward_and_gradient(case):
    c = Case(**case)
    qo, ko = c.out(c.Hq), c.out(c.Hk)
    before = c.fused.clone()
    g.gpd_head_norm_rope(c.q, c.k, c.table, c.pos, qo, ko, c.D, **c.args())
    c.check_forward(qo, ko)
    dqi, dki = c.out(c.Hq), c.out(c.Hk)
    c.backward(dqi, dki)
    c.check_backward(dqi, dki)
    assert torch.equal(before, c.fused)


@pytest.mark.parametrize("case", [CASES[1], CASES[12], CASES[20]])
def test_in_place_leaves_the_same_bits_and_the_values_alone(case):
    c = Case(**case)
    qo, ko = c.out(c.Hq), c.out(c.Hk)
    g.gpd_head_norm_rope(c.q, c.k, c.table, c.pos, qo, ko, c.D, **c.args())
    dqi, dki = c.out(c.Hq), c.out(c.Hk)
    c.backward(dqi, dki)
    dw = c.dw
    dq, dk = c.dq.clone(), c.dk.clone()
    c.backward(c.dq, c.dk)
    assert torch.equal(c.dq, dqi) and torch.equal(c.dk, dki)
    assert not c.norm or (torch.equal(dw[0], c.dw[0]) and torch.equal(dw[1], c.dw[1]))
    c.dq.copy_(dq)
    c.dk.copy_(dk)
    values = c.fused[:, (c.Hq + c.Hk) * c.D:].clone()
    if c.norm:                                         # the gradient over the inputs
        q, k = c.q.clone(), c.k.clone()
        c.backward(c.q, c.k)
        assert torch.equal(c.q, dqi) and torch.equal(c.k, dki)
        c.q.copy_(q)
        c.k.copy_(k)
    g.gpd_head_norm_rope(c.q, c.k, c.table, c.pos, c.q, c.k, c.D, **c.args())
    assert torch.equal(c.q, qo) and torch.equal(c.k, ko) and torch.equal(values, c.fused[:, (c.Hq + c.Hk) * c.D:])


def test_queries_or_keys_alone_and_no_tokens():
    c = Case(T=17, Hq=4, Hk=2, D=128, R=128)
    qo, ko = c.out(4), c.out(2)
    g.gpd_head_norm_rope(c.q, c.k, c.table, c.pos, qo, ko, 128, **c.args())
    q1, k1 = c.out(4), c.out(2)
    g.gpd_head_norm_rope(c.q, None, c.table, c.pos, q1, None, 128, q_weight=c.wq, eps=EPS)
    g.gpd_head_norm_rope(None, c.k, c.table, c.pos, None, k1, 128, k_weight=c.wk, eps=EPS)
    assert torch.equal(q1, qo) and torch.equal(k1, ko)
    dk, dw = c.out(2), torch.empty(128, device="cuda")
    ws = torch.empty(2 * g.GPD_HEAD_NORM_MAX_PARTS * 128, device="cuda")
    g.gpd_head_norm_rope_backward(None, c.dk, None, c.k, c.table, c.pos, None, dk, 128, k_weight=c.wk, dk_weight=dw, workspace=ws)
    ref, size, wref, wsize = backward(c.heads(c.dk), c.heads(c.k), c.wk, c.table, c.pos, None, False)
    check_close(dk, ref.flatten(1), 2 * STEPS, size.flatten(1))
    check_close(dw, wref, 2 * STEPS + 34 * 2.0 ** -24, wsize)
    dw2 = torch.full((128,), 3.0, device="cuda")
    g.gpd_head_norm_rope_backward(c.dq[:0], c.dk[:0], c.q[:0], c.k[:0], c.table, c.pos[:0], qo[:0], dk[:0], 128, q_weight=c.wq,
                                  k_weight=c.wk, dq_weight=dw, dk_weight=dw2, workspace=ws)
    assert not dw.any() and not dw2.any()
    g.gpd_head_norm_rope(c.q[:0], c.k[:0], c.table, c.pos[:0], qo[:0], ko[:0], 128, **c.args())


def test_positions_outside_the_table_and_axes_that_are_none_show_as_nan():
    for R, neighbours in ((128, False), (64, True), (62, False)):
        c = Case(T=6, Hq=2, Hk=1, D=128, R=R, axes=2, neighbours=neighbours, P=50)
        c.axes[3] = 2                                  # there are two
        c.axes[4], c.axes[5] = 0, 1
        c.pos[2, 0], c.pos[3, 1], c.pos[5, 0] = -1, 50, 2 ** 31 - 1
        qo, ko = c.out(2), c.out(1)
        g.gpd_head_norm_rope(c.q, c.k, c.table, c.pos, qo, ko, 128, **c.args())
        outside = (c.pos < 0) | (c.pos >= 50)
        bad = torch.zeros((6, R // 2), dtype=torch.bool, device="cuda")
        for j in range(R // 2):
            a = int(c.axes[j])
            bad[:, j] = outside[:, a] if a < 2 else True
        cols = torch.zeros((6, 128), dtype=torch.bool, device="cuda")
        for j in range(R // 2):
            i, k = (2 * j, 2 * j + 1) if neighbours else (j, j + R // 2)
            cols[:, i] = cols[:, k] = bad[:, j]
        assert torch.equal(torch.isnan(qo).view(6, 2, 128), cols[:, None].expand(6, 2, 128))
        assert torch.equal(torch.isnan(ko), cols)


def test_infinities_in_columns_that_stay_do_not_reach_their_neighbours():
    c = Case(T=3, Hq=2, Hk=1, D=128, R=64, norm=False)
    c.q[1, 70] = math.inf
    c.q[2, 128 + 127] = math.nan
    qo, ko = c.out(2), c.out(1)
    g.gpd_head_norm_rope(c.q, c.k, c.table, c.pos, qo, ko, 128)
    bad = torch.zeros_like(qo, dtype=torch.bool)
    bad[1, 70] = bad[2, 255] = True
    assert torch.equal(~torch.isfinite(qo), bad) and torch.isfinite(ko).all()


def test_zero_heads_and_small_numbers():
    """A head of zeros has s = eps^-1/2 and stays zero; tiny heads are carried by eps."""
    c = Case(T=4, Hq=2, Hk=1, D=128, R=128, type=F32)
    c.q[1] = 0
    c.q[2] *= 1e-20
    qo, ko = c.out(2), c.out(1)
    g.gpd_head_norm_rope(c.q, c.k, c.table, c.pos, qo, ko, 128, **c.args())
    c.check_forward(qo, ko)
    assert not qo[1].any()
    dqi, dki = c.out(2), c.out(1)
    c.backward(dqi, dki)
    c.check_backward(dqi, dki)


def test_gradient_agrees_with_differences():
    c = Case(T=3, Hq=2, Hk=1, D=16, R=12, type=F32, axes=2)
    dqi, dki = c.out(2), c.out(1)
    c.backward(dqi, dki)
    step = 2.0 ** -20

    def loss(q, w):
        return float((forward(q.view(3, 2, 16), w, c.table, c.pos, c.axes, False)[0].flatten(1) * c.dq.double()).sum())
    q, w = c.q.double(), c.wq.double()
    for t, i in ((0, 0), (1, 7), (2, 31), (1, 13)):
        d = torch.zeros_like(q)
        d[t, i] = step
        # second differences of a function whose third derivatives are of order one: the step's square, and FP64's rounding over the step
        assert abs((loss(q + d, w) - loss(q - d, w)) / (2 * step) - float(dqi[t, i])) < 1e-5
    for i in (0, 5, 15):
        d = torch.zeros_like(w)
        d[i] = step
        assert abs((loss(q, w + d) - loss(q, w - d)) / (2 * step) - float(c.dw[0][i])) < 1e-5


def test_far_positions_and_a_long_table():
    """Angles come from 64 bits, whatever the position: position 131071 turned forth and back."""
    table = g.new_rope_table(131072, 64)
    pos = torch.tensor([131071, 100000, 7], device="cuda")
    j = torch.arange(32, dtype=torch.float64)
    for i, p in enumerate(pos.tolist()):
        a = p * 10000.0 ** (-2 * j / 64)
        assert float((table[p].cpu().double() - torch.cat([a.cos(), a.sin()])).abs().max()) < 2.0 ** -24
    x = torch.randn((3, 128), device="cuda")
    y, z = torch.empty_like(x), torch.empty_like(x)
    g.gpd_head_norm_rope(x, None, table, pos, y, None, 64)
    g.gpd_head_norm_rope_backward(y, None, None, None, table, pos, z, None, 64)
    assert not torch.allclose(x, y, atol=0.1) and torch.allclose(x, z, atol=1e-5)


def test_refusals():
    c = Case(T=4, Hq=2, Hk=1, D=128, R=128, axes=2)
    qo, ko = c.out(2), c.out(1)
    ok = dict(q=c.q, k=c.k, table=c.table, positions=c.pos, q_out=qo, k_out=ko, head_dim=128, **c.args())

    def refused(match=None, error=ValueError, **kw):
        with pytest.raises(error, match=match):
            g.gpd_head_norm_rope(**{**ok, **kw})
    refused("heads", head_dim=100)
    refused("head_dim", head_dim=0)
    refused("head_dim", head_dim=512)
    refused("q_out", q_out=None)
    refused("q_out", q_out=ko)
    refused("bfloat16", k=c.k.float())
    refused("axes", axes=None)
    refused("axes", axes=c.axes[:-1])
    refused("positions", positions=None)
    refused("positions", positions=c.pos[:3])
    refused("positions", positions=c.pos.float())
    refused("table", table=None)
    refused("table", table=c.table[:, :127])
    refused("table", table=c.table.double())
    refused("q_weight", q_weight=c.wq[:64])
    refused("one type", q_weight=c.wq.float())
    refused("cuda", k=c.k.cpu())
    refused(error=g.GpdError, q_weight=None)                       # one weight without the other
    refused(error=g.GpdError, table=None, positions=None, axes=None, q_weight=None, k_weight=None)     # nothing to do
    refused(error=g.GpdError, table=torch.zeros((5, 130), device="cuda"), axes=torch.zeros(65, dtype=torch.uint8, device="cuda"))
    odd = torch.zeros((4, 6), device="cuda")
    with pytest.raises(g.GpdError):
        g.gpd_head_norm_rope(odd, None, None, None, odd, None, 3, q_weight=torch.ones(3, device="cuda"))
    dw, ws = torch.empty(128, device="cuda"), torch.empty(2 * g.GPD_HEAD_NORM_MAX_PARTS * 128, device="cuda")
    back = dict(dq=c.dq, dk=c.dk, q=c.q, k=c.k, table=c.table, positions=c.pos, dq_in=qo, dk_in=ko, head_dim=128, dq_weight=dw,
                dk_weight=dw.clone(), workspace=ws, **c.args())
    for kw in (dict(workspace=ws[:-1]), dict(workspace=None), dict(dq_weight=None), dict(q=None), dict(k_weight=None)):
        with pytest.raises(g.GpdError):
            g.gpd_head_norm_rope_backward(**{**back, **kw})
    with pytest.raises(ValueError):
        g.gpd_head_norm_rope_backward(**{**back, "dk_in": None})
