"""Adapters, head norms and clipping on tensors of more than 2^31 elements: offsets of rows do not fit in 32 bits."""

import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

import paper_1811_10751_b200 as g                                          # noqa: E402
from lm_reference import check_close                                       # noqa: E402

BF = torch.bfloat16


@pytest.fixture(autouse=True)
def free_memory():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def _rand(seed, *shape):
    return torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


def _far(rows, cols, values):
    """`values` in rows so far apart that the last begins beyond 2^31 elements."""
    ld = (1 << 31) // (rows - 1) + 4096 & ~63
    m = torch.empty(rows * ld, dtype=BF, device="cuda").view(rows, ld)[:, :cols]
    m.copy_(values)
    assert m.stride(0) * (rows - 1) >= 1 << 31
    return m


@pytest.mark.parametrize("D", [128, 6])                   # with vectors, element by element
def test_heads_in_rows_far_apart(D):
    T, H = 40, 3
    x, w = _far(T, H * D, _rand(1, T, H * D)), (1 + 0.1 * _rand(2, D)).to(BF)
    y = torch.empty_like(x, memory_format=torch.contiguous_format)
    table, pos = g.new_rope_table(64, D), torch.arange(T, device="cuda")
    g.gpd_head_norm_rope(x, None, table, pos, y, None, D, q_weight=w)
    z = x.double().view(T, H, D)
    z = z / torch.sqrt(z.square().mean(2, keepdim=True) + 1e-6) * w.double()
    a, b = z.chunk(2, 2)
    c, s = (t[:, None] for t in table[:T].double().chunk(2, 1))
    check_close(y, torch.cat([a * c - b * s, b * c + a * s], 2).flatten(1), 2.0 ** -19, torch.cat([a.abs() + b.abs()] * 2, 2).flatten(1))
    dx, dw, ws = _far(T, H * D, torch.zeros(())), torch.empty(D, device="cuda"), torch.empty(2 * g.GPD_HEAD_NORM_MAX_PARTS * D, device="cuda")
    g.gpd_head_norm_rope_backward(y, None, x, None, table, pos, dx, None, D, q_weight=w, dq_weight=dw, workspace=ws)
    near = x.contiguous()
    dx2, dw2 = torch.empty_like(near), torch.empty_like(dw)
    g.gpd_head_norm_rope_backward(y, None, near, None, table, pos, dx2, None, D, q_weight=w, dq_weight=dw2, workspace=ws)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)


@pytest.mark.parametrize("lens", [[70, 90], [1] * 40, [40, 3, 17]])
@pytest.mark.parametrize("shift", [0, 1])                 # on 16-byte boundaries, off them
def test_adapters_in_rows_far_apart(lens, shift):
    T, K, N, r, n = sum(lens), 128, 192, 16, 2
    index = torch.arange(len(lens), device="cuda") % n
    offsets = torch.tensor([0] + lens, device="cuda").cumsum(0)
    near = _rand(1, T, K + shift).to(BF)[:, shift:], _rand(2, T, N + shift).to(BF)[:, shift:]
    A, B = (_rand(3, n, r, K) / 11).to(BF), (_rand(4, n, N, r) / 4).to(BF)

    def both(x, base):
        out, h = torch.empty((T, N), dtype=BF, device="cuda"), torch.empty((T, r), device="cuda")
        g.gpd_adapter(x, A, B, offsets, index, out, h, base=base)
        dx, dA, dB = torch.empty((T, K), dtype=BF, device="cuda"), torch.empty((n, r, K), device="cuda"), torch.empty((n, N, r), device="cuda")
        ws = torch.empty(g.gpd_adapter_backward_workspace(T, K, N, n, r), dtype=torch.uint8, device="cuda")
        g.gpd_adapter_backward(base, x, A, B, h, offsets, index, dx, dA, dB, ws, dbase=x)
        return out, h, dx, dA, dB
    want = both(*near)
    far = both(_far(T, K + shift, _rand(1, T, K + shift))[:, shift:], _far(T, N + shift, _rand(2, T, N + shift))[:, shift:])
    assert all(torch.equal(a, b) for a, b in zip(want, far))


def test_gradients_of_more_elements_than_32_bits_count():
    n = (1 << 31) + 12345
    x = torch.zeros(n, dtype=torch.float16, device="cuda")
    at = torch.tensor([0, 1, 8191, 1 << 30, (1 << 31) - 1, 1 << 31, n - 1], device="cuda")
    x[at] = 3.0
    small = torch.full((10,), 2.0, device="cuda")
    norm, ws = torch.empty(1, device="cuda"), torch.empty(g.GPD_GRAD_NORM_WORKSPACE, dtype=torch.uint8, device="cuda")
    g.gpd_grad_norm([x, small], norm, ws)
    assert float(norm) == pytest.approx(math.sqrt(7 * 9 + 40), rel=1e-6)
    g.gpd_clip_grads([x, small], norm, 1.0)
    check_close(x[at], torch.full((7,), 3.0, dtype=torch.float64, device="cuda") / float(norm), 2.0 ** -23)
    assert int(torch.count_nonzero(x)) == 7
