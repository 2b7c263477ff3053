"""More rows of logits than a launch has CTAs in its second dimension (65535): a CTA takes several rows in turn."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

import paper_1811_10751_b200 as g                            # noqa: E402
from tests.lm_reference import check_close                   # noqa: E402

REL = 2e-5                                                   # as in test_gpu_lm_logits.py
GRID = 65535


def _rand(seed, *shape):
    return torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


@pytest.mark.parametrize("K", [100, 1024])
@pytest.mark.parametrize("grad", [True, False])
@pytest.mark.parametrize("which", ["between", "every other", "none"])
def test_distillation_of_many_rows_some_without_weight(K, grad, which):
    """A CTA's first and third row have long lists, the one between them no weight: each row keeps its own list."""
    V, T = 64, 2 * GRID + 2000
    x = _rand(1, T, V)
    ids = torch.randint(0, V, (T, K), device="cuda", dtype=torch.int32, generator=torch.Generator(device="cuda").manual_seed(2))
    t = _rand(3, T, K).bfloat16()
    w = torch.rand(T, device="cuda", generator=torch.Generator(device="cuda").manual_seed(4)) + 0.5
    if which == "between":
        w[GRID:2 * GRID] = 0
    elif which == "every other":
        w[1::2] = 0
    loss, d = torch.full((T,), 9.0, device="cuda"), torch.full_like(x, 9.0) if grad else None
    g.gpd_distill_topk(x, ids, t, w, loss, dlogits=d)
    for r0 in range(0, T, 30000):                            # in 64 bits, some rows at a time
        r = slice(r0, min(T, r0 + 30000))
        logp, logq, wr = torch.log_softmax(x[r].double(), 1), torch.log_softmax(t[r].double(), 1), w[r].double()
        q, at = logq.exp(), ids[r].long()
        ref = (q * (logq - logp.gather(1, at))).sum(1) * wr
        # terms of either sign: log q down to -16, log p down to -12
        assert bool(((loss[r].double() - ref).abs() <= wr * REL * 30).all())
        if grad:
            s = torch.zeros_like(logp).scatter_add_(1, at, q)
            check_close(d[r], (logp.exp() - s) * wr[:, None], REL, (logp.exp() + s) * wr[:, None])
    again, d2 = torch.empty_like(loss), torch.empty_like(x) if grad else None
    for _ in range(3):
        g.gpd_distill_topk(x, ids, t, w, again, dlogits=d2)
        assert torch.equal(loss, again) and (not grad or torch.equal(d, d2))


@pytest.mark.parametrize("K", [0, 5])
def test_log_probabilities_of_many_rows_are_those_of_few(K):
    V, T = 100, 2 * GRID + 77
    x = _rand(1, T, V).bfloat16()
    x[5::7] = x[5::7, :1]                                    # rows of equal entries
    tok = torch.randint(0, V, (T, 2), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))

    def outputs(n):
        return (torch.full((n, 2), 9.0, device="cuda"), torch.full((n,), 9.0, device="cuda"), torch.full((n,), 9.0, device="cuda"),
                torch.full((n, K), -9, device="cuda", dtype=torch.int32), torch.full((n, K), 9.0, device="cuda"))

    def call(rows, o):
        g.gpd_token_logprobs(x[rows], tok[rows], o[0], o[1], entropy=o[2], top_ids=o[3] if K else None, top_logprobs=o[4] if K else None)
    whole = outputs(T)
    call(slice(0, T), whole)
    for r0 in range(0, T, 30000):
        r = slice(r0, min(T, r0 + 30000))
        part = outputs(r.stop - r.start)
        call(r, part)
        assert all(torch.equal(a[r], b) for a, b in zip(whole, part))
    ref = torch.log_softmax(x.double(), 1)
    assert bool(((whole[0].double() - ref.gather(1, tok)).abs() <= REL + 2.0 ** -20 * 8).all())
    assert bool(((whole[2].double() + (ref.exp() * ref).sum(1)).abs() <= REL * 7).all())
