"""8-bit products over long contractions, to 16 bits: the sum's error stays below the result's own rounding.

All operands are positive, so that whatever an addition cuts off adds up.  Bound: the result's rounding, and for the sum that
of test_gpu_lm_gemm.py for FP32 results, (20 + K / 512) 2^-23 of it.  The operands repeat along the contraction, which
makes the 64-bit product a short one."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

import paper_1811_10751_b200 as g                            # noqa: E402
from tests.lm_reference import check_close                   # noqa: E402

E4 = torch.float8_e4m3fn
BF, HF = torch.bfloat16, torch.float16
PERIOD = 8192


def _operand(seed, rows, K, byte):
    """[rows, K] numbers of 1 .. 1.875, all blocks with the scale 2^(byte - 127), and the values of one period."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    base = (torch.randint(8, 16, (rows, PERIOD), device="cuda", generator=gen).float() / 8).to(E4)
    q, s = g.new_fp8(rows, K, E4, 1)
    q.view(torch.uint8).view(rows, K // PERIOD, PERIOD).copy_(base.view(torch.uint8)[:, None, :].expand(rows, K // PERIOD, PERIOD))
    s.view(torch.uint8).fill_(byte)
    return q, s, base.double() * 2.0 ** (byte - 127)


# tiles that fill the GPU without splitting the contraction, wide tiles of CTA pairs, and a split contraction
@pytest.mark.parametrize("M,N,K", [(800, 800, 2 ** 18), (800, 800, 2 ** 20), (1300, 1100, 2 ** 18), (24, 40, 2 ** 20), (3, 2000, 2 ** 19)])
@pytest.mark.parametrize("out", [HF, BF])
def test_sum_of_a_long_contraction(M, N, K, out):
    A, sa, a = _operand(1, M, K, 127 - 8)
    B, sb, b = _operand(2, N, K, 127)
    ref = (a @ b.t()) * (K // PERIOD)
    D = torch.empty((M, N), dtype=out, device="cuda")
    g.gpd_gemm_fp8(A, sa, B, sb, D)
    assert g.gpd_device_status() == 0
    check_close(D, ref, (20 + K / 512) * 2.0 ** -23)
    prev = ref.to(out)
    D.copy_(prev)
    g.gpd_gemm_fp8(A, sa, B, sb, D, accumulate=True)
    check_close(D, ref + prev.double(), (20 + K / 512) * 2.0 ** -23)
