"""Distillation from lists with infinities and with ids beyond the row."""

import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

import paper_1811_10751_b200 as g                            # noqa: E402
from tests.lm_reference import check_close                   # noqa: E402

BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32
REL = 2e-5                                                   # as in test_gpu_lm_logits.py


def _rand(seed, *shape):
    return torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


def _lists(T, V, K, seed=5):
    """Ids without repetition in a row."""
    return torch.argsort(_rand(seed, T, V), dim=1)[:, :K].int().contiguous()


@pytest.mark.parametrize("V", [300, 40000])
@pytest.mark.parametrize("dtype,ttype", [(F32, F32), (BF, HF), (HF, BF)])
@pytest.mark.parametrize("tau", [1.0, 2.0])
def test_teacher_logit_of_infinity(V, dtype, ttype, tau):
    """softmax over a list with +inf is NaN: so are the loss and the gradient at the list's ids; elsewhere it is w tau p."""
    T, K = 6, 40
    x, t, ids = _rand(1, T, V).to(dtype), _rand(2, T, K).to(ttype), _lists(T, V, K)
    w = torch.linspace(0.5, 1.5, T, device="cuda")
    t[0, 3] = math.inf
    t[1, :] = math.inf
    t[2, 7], t[2, 9] = math.inf, -math.inf
    t[3, K - 1], w[3] = math.inf, 0.0                        # no weight: not read
    t[4, 5], ids[4, 5] = math.inf, -1                        # does not count
    loss, d = torch.full((T,), 5.0, device="cuda"), torch.full_like(x, 5.0)
    g.gpd_distill_topk(x, ids, t, w, loss, dlogits=d, temperature=tau)
    alone = torch.full((T,), 5.0, device="cuda")
    g.gpd_distill_topk(x, ids, t, w, alone, temperature=tau)
    p = torch.softmax(x.double() / tau, 1) * (w.double() * tau)[:, None]
    for r in (0, 1, 2):
        assert math.isnan(float(loss[r])) and math.isnan(float(alone[r])), (r, float(loss[r]))
        listed = torch.zeros(V, dtype=torch.bool, device="cuda")
        listed[ids[r].long()] = True
        assert bool(torch.isnan(d[r][listed]).all())
        check_close(d[r][~listed][None], p[r][~listed][None], REL)
    assert float(loss[3]) == 0 and bool((d[3] == 0).all())
    assert bool(torch.isfinite(loss[4:]).all()) and bool(torch.isfinite(d[4:]).all()) and torch.equal(loss[3:], alone[3:])


@pytest.mark.parametrize("V", [300, 40000])
@pytest.mark.parametrize("index", [torch.int32, torch.int64])
def test_id_beyond_the_row_shows_in_the_gradient_too(V, index):
    T, K = 5, 9
    x, t, ids = _rand(1, T, V), _rand(2, T, K), _lists(T, V, K).to(index)
    ids[0, 4] = V
    ids[1, :] = V + 5
    ids[2, 8] = 2 ** 31 - 1 if index == torch.int32 else 2 ** 40
    x[2] = -math.inf
    ids[3, 2], w = V, torch.ones(T, device="cuda")
    w[3] = 0.0                                               # no weight: not read
    loss, d = torch.full((T,), 5.0, device="cuda"), torch.full_like(x, 5.0)
    g.gpd_distill_topk(x, ids, t, w, loss, dlogits=d)
    for r in (0, 1, 2):
        assert math.isnan(float(loss[r])) and bool(torch.isnan(d[r]).all()), r
    assert float(loss[3]) == 0 and bool((d[3] == 0).all())
    assert math.isfinite(float(loss[4])) and bool(torch.isfinite(d[4]).all())


def test_masked_row_with_a_bad_list():
    """Neither softmax exists: NaN, not the 0 that a masked row with a sound list gets."""
    x, t, ids = torch.full((3, 500), -math.inf, device="cuda"), _rand(2, 3, 9), _lists(3, 500, 9)
    t[0, 2], t[1, 2] = math.inf, math.nan
    loss, d = torch.full((3,), 5.0, device="cuda"), torch.full_like(x, 5.0)
    g.gpd_distill_topk(x, ids, t, None, loss, dlogits=d)
    for r in (0, 1):
        assert math.isnan(float(loss[r])) and bool(torch.isnan(d[r]).all())
    assert float(loss[2]) == math.inf and bool((d[2] == 0).all())
