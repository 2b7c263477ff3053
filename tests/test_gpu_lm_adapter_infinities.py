"""Infinities in x, where the rank is no multiple of the tensor cores' steps: what stands behind the rank adds nothing to them."""

import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

from test_gpu_lm_adapters import BF16, F16, F32, Case          # noqa: E402


@pytest.mark.parametrize("type,out_type", [(BF16, BF16), (BF16, F32), (F16, F16), (F16, F32)])
@pytest.mark.parametrize("r", [1, 7, 8, 24, 40, 100])
@pytest.mark.parametrize("lens,pad", [([1, 2, 1, 16, 3], 0), ([40, 30, 25], 0), ([40, 30, 25], 1), ([1, 2, 1, 16, 3], 1)],
                         ids=["single", "long", "long, off boundaries", "single, off boundaries"])
def test_results_are_infinite_where_the_formula_is(type, out_type, r, lens, pad):
    c = Case(lens=lens, index=[i % 2 for i in range(len(lens))], n=2, r=r, K=136, N=72, type=type, out=out_type, pad=pad, offset=pad)
    c.A.copy_(c.A.abs() + 0.25)                                # every number of h is infinite with x's sign, every one of B positive
    c.B.copy_(c.B.abs() + 0.25)
    c.x[0, 3], c.x[c.T - 1, 130] = math.inf, -math.inf
    out, h = c.forward()
    for row, v in ((0, math.inf), (c.T - 1, -math.inf)):
        assert bool((h[row] == v).all()) and bool((out[row] == v).all())
    rest = slice(1, c.T - 1)
    assert torch.isfinite(out[rest]).all() and torch.isfinite(h[rest]).all()
