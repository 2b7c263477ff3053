"""Gradient of the norms per head where the inputs are far from one, against the formulas in 64 bits."""

import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

import paper_1811_10751_b200 as g                              # noqa: E402
from lm_reference import check_close                           # noqa: E402
from test_gpu_lm_heads import BF16, F32, STEPS, Case, turn     # noqa: E402


@pytest.mark.parametrize("type", [BF16, F32])
@pytest.mark.parametrize("pad", [0, 1])                        # whole vectors, element by element
@pytest.mark.parametrize("size,eps", [(1e15, 1e-6), (1e13, 1e-36), (1e-14, 1e-36), (1e-17, 1e-36), (1e13, 0.0), (1e-14, 0.0),
                                      (1e-17, 0.0), (1.0, 0.0)])
def test_heads_of_any_size(type, pad, size, eps):
    """dx is of the size of dy / x, whatever x is: neither term of it may be lost on the way."""
    c = Case(T=50, Hq=5, Hk=2, D=128, R=64, type=type, pad=pad)
    c.fused.mul_(size)
    dqi, dki = c.out(5), c.out(2)
    dw, ws = [torch.full((128,), math.nan, device="cuda") for _ in range(2)], torch.empty(2 * g.GPD_HEAD_NORM_MAX_PARTS * 128, device="cuda")
    g.gpd_head_norm_rope_backward(c.dq, c.dk, c.q, c.k, c.table, c.pos, dqi, dki, 128, dq_weight=dw[0], dk_weight=dw[1], workspace=ws,
                                  **(c.args() | {"eps": eps}))
    for x, dy, w, o, d in ((c.q, c.dq, c.wq, dqi, dw[0]), (c.k, c.dk, c.wk, dki, dw[1])):
        x, w = c.heads(x).double(), w.double()
        gr, gsize = turn(c.heads(dy).double(), c.table, c.pos, None, False, back=True)
        s = 1 / torch.sqrt(x.square().mean(2, keepdim=True) + eps)
        n = x * s
        dx = s * (gr * w - n * (gr * w * n).mean(2, keepdim=True))
        dsize = s * (gsize * w.abs() + n.abs() * (gsize * w.abs() * n.abs()).mean(2, keepdim=True))
        check_close(o, dx.flatten(1), 2 * STEPS, dsize.flatten(1))
        check_close(d, (gr * n).sum((0, 1)), 2 * STEPS + c.T * x.shape[1] * 2.0 ** -24, (gsize * n.abs()).sum((0, 1)))
