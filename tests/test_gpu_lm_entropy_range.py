"""Entropy of rows whose logits lie further apart than the largest FP32 number: the difference of a masked entry to the row's
maximum overflows, its share of the entropy is 0 all the same."""

import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

import paper_1811_10751_b200 as g                            # noqa: E402


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,K", [(9, 3), (5000, 3), (5000, 0), (70001, 3), (300000, 3), (300000, 0)])
def test_masks_of_the_lowest_value_beside_huge_logits(dtype, V, K):
    """Two equal maxima of 1e37 and masks: the probabilities are 1/2 and 0, the entropy ln 2.  2e-5: as for other rows."""
    x = torch.full((3, V), torch.finfo(dtype).min, device="cuda", dtype=dtype)
    x[0, 1] = x[0, V - 2] = 1e37
    x[1, 1] = x[1, V - 2] = 1e37
    x[1, 4] = -math.inf
    x[2, 3] = 1e37
    tok = torch.tensor([1, V - 2, 3], device="cuda")
    lp, lse, H = (torch.empty(3, device="cuda") for _ in range(3))
    ids = torch.empty((3, K), device="cuda", dtype=torch.int32) if K else None
    g.gpd_token_logprobs(x, tok, lp, lse, entropy=H, top_ids=ids)
    want = torch.tensor([math.log(2), math.log(2), 0.0], device="cuda")
    assert bool(((H - want).abs() < 2e-5).all()), H.tolist()
    if K:
        assert ids[:, 0].tolist() == [1, 1, 3] and ids[:2, 1].tolist() == [V - 2, V - 2]
