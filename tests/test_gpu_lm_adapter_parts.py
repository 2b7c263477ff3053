"""What adapters' products keep of FP32 factors whose numbers differ widely in size: the large ones meet zeros, so that only what is
kept of the small ones counts."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

from lm_reference import HALF_ULP, TINY                        # noqa: E402
from test_gpu_lm_adapters import BF16, F16, F32, STEP, Case    # noqa: E402



def check(got, ref, lost):
    """`lost`: before the result's one rounding."""
    bound = lost + ref.abs() * HALF_ULP[got.dtype] * (1 + 1e-6) + TINY[got.dtype]
    d = (got.double() - ref).abs()
    assert bool((d <= bound).all()), float((d / bound).max())


# aligned rows and long segments, rows off 16-byte boundaries, single rows
FORMS = {"long": dict(lens=[130, 70]), "off boundaries": dict(lens=[130, 70], pad=1, offset=1), "single": dict(lens=[1, 1, 2, 1] * 5)}
# of a large number's size, what is lost of those far below it (2^-39 of each part's row, or of a column of three parts)
FAR = 3 * 2.0 ** -39


def case(form, type, out=F32, r=3, N=136, K=264):
    f = FORMS[form]
    return Case(index=[i % 2 for i in range(len(f["lens"]))], n=2, r=r, K=K, N=N, type=type, out=out, **f)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("type", [BF16, F16])
def test_small_numbers_of_a_row_beside_a_large_one(form, type):
    """FP32 results: 24 bits of h.  One step of the tensor cores for each of the three parts (a rank of 3 is one step deep)."""
    c = case(form, type)
    c.A[:, 0] *= 1024
    c.A[:, 1:] /= 8
    c.B[:, :, 0] = 0
    out, h = c.forward(base=None)
    assert float(h[:, 0].abs().median()) > 1000 * float(h[:, 1:].abs().median())
    for a, b, i in c.segments:
        s, B, hd = float(c.scale[i]), c.B[i].double(), h[a:b].double()
        top = hd.abs().amax(1, keepdim=True)
        size = s * (hd.abs() @ B.abs().t())
        check(out[a:b], s * (hd @ B.t()), (3 * STEP + 2.0 ** -23) * size + FAR * s * top * B.abs().sum(1))


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("type", [BF16, F16])
def test_small_gradients_of_a_row_beside_a_large_one(form, type):
    """The same of u in the gradient of the input, whose own sums over N lose their part."""
    c = case(form, type)
    c.B[:, :, 0] *= 1024
    c.B[:, :, 1:] /= 8
    c.A[:, 0] = 0
    _, h = c.forward()
    c.backward(h, dbase=None)
    lost_u = 4 * STEP + (c.N / 64 + 16) * 2.0 ** -24
    for a, b, i in c.segments:
        s, A, B, d = float(c.scale[i]), c.A[i].double(), c.B[i].double(), c.dout[a:b].double()
        u, us = s * (d @ B), s * (d.abs() @ B.abs())
        check(c.dx[a:b], u @ A, (lost_u + 3 * STEP + 2.0 ** -23) * (us @ A.abs()) + FAR * us.amax(1, keepdim=True) * A.abs().sum(0))


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("type", [BF16, F16])
def test_small_numbers_of_a_column_beside_a_large_one(form, type):
    """FP32 gradients: 24 bits of h and u.  A chain of 64 rows is 4 steps deep, for three parts 12; then FP32 additions."""
    c = case(form, type)
    _, h = c.forward()
    for first in {i: a for a, _, i in reversed(c.segments)}.values():        # an adapter's first row: large in h where dout is 0
        h[first] *= 131072
        c.dout[first] = 0
    c.backward(h)
    dB, size, top = (torch.zeros(c.B.shape, dtype=torch.float64, device="cuda") for _ in range(3))
    for a, b, i in c.segments:
        d, hd, s = c.dout[a:b].double(), h[a:b].double(), float(c.scale[i])
        dB[i] += s * d.t() @ hd
        size[i] += s * d.abs().t() @ hd.abs()
        top[i] += s * d.abs().sum(0)[:, None]
    for i in range(2):
        top[i] *= torch.cat([h[a:b] for a, b, j in c.segments if j == i]).abs().amax(0).double()
    check(c.dB, dB, (12 * STEP + (c.T / 64 + 8) * 2.0 ** -24) * size + FAR * top)

    c = case(form, type)
    _, h = c.forward()
    for first in {i: a for a, _, i in reversed(c.segments)}.values():        # large in u where x is 0
        c.dout[first] *= 8192
        c.x[first] = 0
    c.backward(h)
    lost_u = 4 * STEP + (c.N / 64 + 16) * 2.0 ** -24
    dA, size, top, most = (torch.zeros(c.A.shape, dtype=torch.float64, device="cuda") for _ in range(4))
    for a, b, i in c.segments:
        d, x, B, s = c.dout[a:b].double(), c.x[a:b].double(), c.B[i].double(), float(c.scale[i])
        u, us = s * (d @ B), s * (d.abs() @ B.abs())
        dA[i] += u.t() @ x
        size[i] += us.t() @ x.abs()
        top[i] += x.abs().sum(0)
        most[i] = torch.maximum(most[i], us.amax(0)[:, None])
    check(c.dA, dA, (lost_u + 12 * STEP + (c.T / 64 + 8) * 2.0 ** -24) * size + FAR * top * most)


# 16-bit results: of a term, what the parts of its FP32 factor lose (nothing of three BF16 parts, 2^-23 of two FP16 ones) and the steps
# of the tensor cores that have more than zeros to add, one for each part
CANCEL = {BF16: 2.0 ** -24 + 3 * STEP, F16: 2.0 ** -22 + 2 * STEP}


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("type", [BF16, F16])
def test_sixteen_bit_results_of_terms_that_cancel(form, type):
    """Two numbers of h (and of u) that are nearly alike, one of them subtracted: the difference is rounded once."""
    c = case(form, type, out=type, r=2)
    c.A[:, 1] = c.A[:, 0]
    c.A[:, 1, 7] *= 1.03125
    c.B[:, :, 1] = -c.B[:, :, 0]
    out, h = c.forward(base=None)
    assert float((h[:, 0] - h[:, 1]).abs().median()) < float(h.abs().median()) / 256
    for a, b, i in c.segments:
        s, B, hd = float(c.scale[i]), c.B[i].double(), h[a:b].double()
        check(out[a:b], s * (hd @ B.t()), (CANCEL[type] + 2.0 ** -23) * s * (hd.abs() @ B.abs().t()))

    c = case(form, type, out=type, r=2)
    c.B[:, :, 1] = c.B[:, :, 0]
    c.B[:, 7, 1] *= 1.03125
    c.A[:, 1] = -c.A[:, 0]
    c.backward(h, dbase=None)
    lost_u = 4 * STEP + (c.N / 64 + 16) * 2.0 ** -24
    for a, b, i in c.segments:
        s, A, B, d = float(c.scale[i]), c.A[i].double(), c.B[i].double(), c.dout[a:b].double()
        u, us = s * (d @ B), s * (d.abs() @ B.abs())
        check(c.dx[a:b], u @ A, lost_u * (us @ A.abs()) + (CANCEL[type] + 2.0 ** -23) * (u.abs() @ A.abs()))


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("type", [BF16, F16])
def test_sixteen_bit_gradients_of_rows_that_cancel(form, type):
    """Two rows with nearly the same h and the opposite gradients, all others without: dB is rounded once."""
    c = case(form, type)
    c.grad = type
    _, h = c.forward()
    pairs = []
    for i in range(2):
        rows = [t for a, b, j in c.segments if j == i for t in range(a, b)]
        c.dout[rows[2:]] = 0
        c.dout[rows[1]] = -c.dout[rows[0]]
        h[rows[1]] = h[rows[0]] * (1 - 2.0 ** -11)
        pairs.append(rows[:2])
    c.backward(h)
    for i, (t, u) in enumerate(pairs):
        d, s = c.dout[t].double()[:, None], float(c.scale[i])
        size = s * d.abs() * (h[t].abs() + h[u].abs()).double()
        check(c.dB[i], s * d * (h[t].double() - h[u].double()), (CANCEL[type] + 2 * 2.0 ** -24) * size)
