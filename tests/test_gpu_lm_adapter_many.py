"""Gradients of more adapters than a grid's second dimension counts."""

import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

import paper_1811_10751_b200 as g                              # noqa: E402
from test_gpu_lm_adapters import BF16, Case                    # noqa: E402


def test_gradients_of_seventy_thousand_adapters():
    n = 70000
    c = Case(lens=[40, 65, 20], index=[n - 1, 3, 65536], n=n, r=4, K=16, N=8, type=BF16)
    _, h = c.forward()
    c.backward(h)
    c.check_backward(h)
    assert g.gpd_device_status() == 0


def test_refused_where_runs_are_counted():
    n = 70000
    c = Case(lens=[1, 2, 1], index=[n - 1, 3, 65536], n=n, r=4, K=16, N=8, type=BF16)
    _, h = c.forward()
    ws = c.workspace()
    before = ws.clone()
    dA, dB, dx = torch.zeros(c.A.shape, device="cuda"), torch.zeros(c.B.shape, device="cuda"), torch.full_like(c.x, math.pi)
    with pytest.raises(g.GpdError):
        g.gpd_adapter_backward(c.dout, c.x, c.A, c.B, h, c.offsets, c.index, dx, dA, dB, ws)
    assert torch.equal(ws, before) and bool((dx == dx[0, 0]).all())            # before anything is launched
    g.gpd_adapter_backward(c.dout, c.x, c.A, c.B, h, c.offsets, c.index, dx, None, None, ws)
