"""Entropy and its gradient where logits are masked, against 64 bits: a masked entry has p = 0, and p log p, p (log p + H)
are 0 there, whatever the upstream gradients, the temperature and the mask's value (-inf or the type's lowest)."""

import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

import paper_1811_10751_b200 as g                            # noqa: E402
from tests.lm_reference import check_close                   # noqa: E402

BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32
REL = 2e-5                                                   # sums and probabilities, as in test_gpu_lm_logits.py


def _rand(seed, *shape):
    return torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("mask", ["inf", "lowest"])
@pytest.mark.parametrize("dentropy", [3.0, -3.0, 1e3, -1e3])
@pytest.mark.parametrize("tau", [0.5, 0.7, 1.0])
@pytest.mark.parametrize("tokens", [True, False])
def test_gradient_of_the_entropy_at_masked_entries(dtype, mask, dentropy, tau, tokens):
    T, V = 4, 1201
    x = (_rand(1, T, V) * 2).to(dtype)
    masked = _rand(2, T, V) < 0.3
    masked[0, 5], masked[1, 7] = True, False
    x[masked] = -math.inf if mask == "inf" else torch.finfo(dtype).min
    tok = torch.tensor([5, 7, 1200, 0], device="cuda")       # the first one is a masked entry
    tau = float(torch.tensor(tau))                           # the FP32 number the kernel sees
    z = x.double() / tau
    lse = torch.logsumexp(z, 1, keepdim=True)
    p = (z - lse).exp()
    logp = torch.where(masked, 0.0, z - lse)                 # p is 0 there (exp(-65504 - lse) too)
    assert bool((p[masked] == 0).all())
    H = -(p * logp).sum(1, keepdim=True)
    gh = torch.full((T,), dentropy, device="cuda")
    gl = _rand(3, T) if tokens else None
    d = torch.full_like(x, 7.0)
    g.gpd_token_logprobs_backward(x, tok, lse[:, 0].float(), H[:, 0].float(), gl, gh, d, temperature=tau)
    a = gl.double()[:, None] if tokens else torch.zeros((T, 1), device="cuda", dtype=torch.float64)
    one = torch.zeros_like(z).scatter_(1, tok[:, None], 1.0)
    ref = (a * (one - p) - dentropy * p * (logp + H)) / tau
    # z - lse is a difference of FP32 numbers: its error goes by their size
    size = torch.where(masked, 0.0, z).abs() + lse.abs() + H
    size = (a.abs() * (one + p) + abs(dentropy) * p * size) / tau
    assert bool(torch.isfinite(d).all())
    check_close(d, ref, REL + 2.0 ** -20 * float(torch.where(masked, 0.0, z).abs().max()), size)
