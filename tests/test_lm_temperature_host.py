"""CPU-only: temperatures that the logit operators refuse, before they would touch a GPU."""

import ctypes as C

import pytest

pytest.importorskip("torch")
import paper_1811_10751_b200 as g            # noqa: E402

P = C.c_void_p(4096)                          # never dereferenced: the checks come first
L = g.lib
# 1e-39 is above 0 but log2(e) / 1e-39 is no FP32 number: every 2^((x - m) / tau) would be 2^(0 * inf)
REFUSED = [0.0, -1.0, float("inf"), float("nan"), 1e-39, 1e-45, 4e-39]


@pytest.mark.parametrize("tau", REFUSED)
def test_temperatures_without_a_finite_reciprocal_are_refused(tau):
    assert L.gpd_token_logprobs(1, P, 100, 4, P, 1, tau, P, P, None, 0, None, None, 2, 100, None) == g.GPD_ERR_ARG
    assert L.gpd_token_logprobs_backward(1, P, 100, 4, P, 1, tau, P, None, P, None, P, 100, 2, 100, None) == g.GPD_ERR_ARG
    assert L.gpd_distill_topk(1, P, 100, 4, P, 8, 0, P, 8, 8, None, tau, P, None, 0, 2, 100, None) == g.GPD_ERR_ARG


@pytest.mark.parametrize("tau", [5e-39, 1e-30, 1e-5, 1.0, 1e30])
def test_other_temperatures_are_not(tau):
    assert L.gpd_token_logprobs(1, None, 100, 4, P, 1, tau, P, P, None, 0, None, None, 0, 100, None) == g.GPD_OK
    assert L.gpd_distill_topk(1, None, 100, 4, P, 8, 0, P, 8, 8, None, tau, P, None, 0, 0, 100, None) == g.GPD_OK
