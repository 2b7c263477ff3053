"""Adapters' second product over many ragged segments: every CTA goes from whole tiles to the ragged ends of segments, and on to the
next tile, many times while its ring of stages turns and what it has written is still leaving."""

import random

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

import paper_1811_10751_b200 as g                              # noqa: E402
from test_gpu_lm_adapters import Case                          # noqa: E402

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def lens(T, seed):
    """Lengths that end at every place in a tile of 64 rows and in a warp's 16, a few of them without rows."""
    rng, out = random.Random(seed), []
    while sum(out) < T:
        out.append(rng.choice([0, 1, 16, 64, 80, 128, rng.randint(17, 63), rng.randint(65, 127), rng.randint(129, 400)]))
    return out


@pytest.mark.parametrize("type,out", [(BF16, BF16), (BF16, F32), (F16, F16), (F16, F32)])
@pytest.mark.parametrize("r", [16, 64, 128])
def test_results_leave_before_their_stages_are_filled_again(type, out, r):
    rows = lens(60000, r)
    rng = random.Random(7)
    c = Case(rows, [rng.randrange(-1, 5) for _ in rows], 5, r, 128, 1096, type, out, seed=r, before=5, behind=9)
    first, h = c.forward()
    c.check_forward(first, h)
    for _ in range(6):
        again, h2 = c.forward()
        assert torch.equal(again, first) and torch.equal(h2, h)
    base = c.base.clone()
    c.forward(out=c.base)                                      # in place: what is read next to what is written
    assert torch.equal(c.base[5:c.T - 9], first[5:c.T - 9])
    assert torch.equal(c.base[:5], base[:5]) and torch.equal(c.base[c.T - 9:], base[c.T - 9:])
    assert g.gpd_device_status() == 0


@pytest.mark.parametrize("type,out", [(BF16, BF16), (F16, F32)])
def test_gradient_of_the_input_likewise(type, out):
    rows = lens(60000, 3)
    rng = random.Random(8)
    c = Case(rows, [rng.randrange(-1, 3) for _ in rows], 3, 64, 1096, 136, type, out, seed=3, before=70, behind=3)
    _, h = c.forward()
    c.backward(h)
    c.check_backward(h)
    dx, dA, dB = c.dx, c.dA, c.dB
    for _ in range(6):
        c.backward(h)
        assert torch.equal(c.dx, dx) and torch.equal(c.dA, dA) and torch.equal(c.dB, dB)
    assert g.gpd_device_status() == 0
