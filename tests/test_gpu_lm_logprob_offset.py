"""Log probabilities do not lose digits to a common offset of a row's logits or to a low temperature.

(x - m) / tau - log s: x - m is exact for neighbours of a factor of two and otherwise off by 2^-24 of itself, the
product with 1 / tau adds 2^-23 of it; log s is off by 2e-5 at most (test_gpu_lm_logits.py).  Nothing grows with m."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

import paper_1811_10751_b200 as g                            # noqa: E402

REL = 2e-5


def _rand(seed, *shape):
    return torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


@pytest.mark.parametrize("offset", [0.0, 1e3, -1e3, 1e5])
@pytest.mark.parametrize("tau", [0.05, 1.0])
@pytest.mark.parametrize("T,V,K", [(5, 900, 20), (3, 40000, 20), (200, 5000, 0)])
def test_offset_and_low_temperature(offset, tau, T, V, K):
    x = _rand(1, T, V) + offset
    tok = torch.randint(0, V, (T,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    x[0, tok[0]] = offset + 12.0                             # all but certain
    lp, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    ids = torch.empty((T, K), device="cuda", dtype=torch.int32) if K else None
    tlp = torch.empty((T, K), device="cuda") if K else None
    g.gpd_token_logprobs(x, tok, lp, lse, top_ids=ids, top_logprobs=tlp, temperature=tau)
    tau = float(torch.tensor(tau))                           # the FP32 number the kernel sees
    z = x.double() / tau
    logp = torch.log_softmax(z, 1)
    bound = REL + 2.0 ** -22 * (z.amax(1, keepdim=True) - z)

    def check(got, at):
        far = (got.double() - logp.gather(1, at)).abs() / bound.gather(1, at)
        assert bool((far <= 1).all()), float(far.max())
        assert bool((got <= 0).all())                        # s holds its largest term, which is 1
    check(lp[:, None], tok[:, None])
    if K:
        check(tlp, ids.long())
