"""Gradients of adapters and 8-bit products, which both hold tensor memory, behind one another on two streams at once."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

import paper_1811_10751_b200 as g                              # noqa: E402
from test_gpu_lm_adapters import BF16, Case               # noqa: E402


def product(M, N, K, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    a, a_scales = g.new_fp8(M, K)
    b, b_scales = g.new_fp8(N, K, block_rows=128)
    g.gpd_quantize_blocks(torch.randn(M, K, device="cuda", generator=gen), q=a, scales=a_scales)
    g.gpd_quantize_blocks(torch.randn(N, K, device="cuda", generator=gen), q=b, scales=b_scales, block_rows=128)
    out = torch.zeros(M, N, device="cuda", dtype=BF16)
    return lambda: g.gpd_gemm_fp8(a, a_scales, b, b_scales, out), out


@pytest.mark.parametrize("r", [16, 64, 128])
def test_gradients_and_products_on_two_streams(r):
    runs, outs = [], []
    for seed in range(2):
        c = Case(lens=[700, 300, 1100], index=[0, 2, 1], n=3, r=r, K=1024, N=1536, type=BF16, seed=seed)
        _, h = c.forward()
        dA, dB, ws = torch.zeros(c.A.shape, device="cuda"), torch.zeros(c.B.shape, device="cuda"), c.workspace()
        first, p = product(2048, 2048, 512, seed)
        second, q = product(130, 640, 2048, seed + 5)

        def run(c=c, h=h, dA=dA, dB=dB, ws=ws, first=first, second=second):
            first()
            g.gpd_adapter_backward(c.dout, c.x, c.A, c.B, h, c.offsets, c.index, None, dA, dB, ws, scale=c.scale)
            second()                                   # right behind the factors' gradients
        runs.append(run)
        outs.append((dA, dB, p, q))
    for run in runs:
        run()
    torch.cuda.synchronize()
    want = [[t.clone() for t in o] for o in outs]
    streams = [torch.cuda.Stream() for _ in runs]
    for _ in range(50):
        for run, st in zip(runs, streams):
            with torch.cuda.stream(st):
                run()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for o, w in zip(outs, want) for a, b in zip(o, w))
    assert g.gpd_device_status() == 0
