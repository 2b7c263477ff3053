"""Clipping of gradients whose dimensions are in another order than usual."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

import paper_1811_10751_b200 as g                              # noqa: E402


def test_dimensions_of_one_element_have_any_stride():
    x = torch.arange(24.0, device="cuda").as_strided((6, 4, 1), (1, 6, 999))   # columns first, as a transposed weight's gradient is
    y = torch.arange(24.0, device="cuda").as_strided((1, 4, 6), (5, 1, 4))
    norm = torch.full((1,), 4.0, device="cuda")
    ox, oy = torch.zeros(24, device="cuda").as_strided((6, 4, 1), (1, 6, 1)), torch.zeros(24, device="cuda").as_strided((1, 4, 6), (24, 1, 4))
    g.gpd_clip_grads([x, y], norm, 1.0, out=[ox, oy])
    assert torch.equal(ox, x / 4) and torch.equal(oy, y / 4)
    e = torch.zeros((0, 4, 3), device="cuda")
    g.gpd_clip_grads([e], norm, 1.0, out=[torch.zeros((3, 4, 0), device="cuda").permute(2, 1, 0)])


def test_other_orders_are_refused():
    x = torch.zeros((6, 4), device="cuda")
    norm = torch.ones(1, device="cuda")
    with pytest.raises(ValueError, match="order"):
        g.gpd_clip_grads([x], norm, 1.0, out=[torch.zeros((4, 6), device="cuda").t()])
