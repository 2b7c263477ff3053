"""Clipping of gradients far above the bound: the factor is below what FP32 holds in 24 bits."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

import paper_1811_10751_b200 as g                              # noqa: E402
from lm_reference import check_close                           # noqa: E402

F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("type", [F32, BF16])
@pytest.mark.parametrize("size,bound", [(1e30, 1e-9), (1e35, 1e-8), (1e35, 1e-3), (1e36, 1e-12), (1e20, 1e-30), (1e3, 1e-36)])
def test_one_rounding_whatever_the_factor(type, size, bound):
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = (torch.randn(10007, device="cuda", generator=gen) * size).to(type)
    x[::7] *= 2.0 ** -60                                       # beside the others nothing: zero, or what FP32 has of it
    norm, ws = torch.empty(1, device="cuda"), torch.empty(g.GPD_GRAD_NORM_WORKSPACE, dtype=torch.uint8, device="cuda")
    g.gpd_grad_norm([x], norm, ws)
    want = x.double() * (bound / float(norm))
    out = torch.empty(10007, device="cuda")
    g.gpd_clip_grads([x], norm, bound, out=[out])
    check_close(out, want, 2 * 2.0 ** -24)
    g.gpd_clip_grads([x], norm, bound)
    check_close(x, want, 2 * 2.0 ** -24)
