"""Batches as a server has them, long prompts beside single tokens, and gradients of every type in a graph."""

import random

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

import paper_1811_10751_b200 as g                              # noqa: E402
from test_gpu_lm_adapters import BF16, F16, F32, Case          # noqa: E402


@pytest.mark.parametrize("long,single", [([4000], 300), ([4000], 200), ([1500, 17, 700], 130), ([], 300), ([33] * 20, 20)])
@pytest.mark.parametrize("type,out,r", [(BF16, BF16, 16), (F16, F32, 64), (BF16, F32, 7), (F16, F16, 128)])
def test_prompts_beside_single_tokens(long, single, type, out, r):
    rng = random.Random(len(long) + single)
    lens = long + [1] * single
    rng.shuffle(lens)
    c = Case(lens, [rng.randrange(-1, 9) for _ in lens], 9, r, 264, 328, type, out, seed=single, before=1, behind=2)
    o, h = c.forward()
    c.check_forward(o, h)
    c.backward(h)
    c.check_backward(h)
    assert g.gpd_device_status() == 0


@pytest.mark.parametrize("lens", [[500, 300, 700], [3, 1, 2, 1, 5]])
@pytest.mark.parametrize("type,grad", [(F16, F16), (F16, F32), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradients_in_a_graph(lens, type, grad, accumulate):
    """FP16's maxima are set to zero between launches that follow each other closely; accumulated gradients grow with every replay."""
    c = Case(lens, [i % 3 for i in range(len(lens))], 3, 24, 264, 328, type, grad=grad)
    _, h = c.forward()
    dx, ws = torch.zeros_like(c.dbase), c.workspace()
    dA, dB = (torch.zeros(s, device="cuda", dtype=grad) for s in (c.A.shape, c.B.shape))

    def run():
        g.gpd_adapter_backward(c.dout, c.x, c.A, c.B, h, c.offsets, c.index, dx, dA, dB, ws, dbase=c.dbase, scale=c.scale, accumulate=accumulate, stream=st)
    st, results = torch.cuda.Stream(), (dx, dA, dB)
    torch.cuda.synchronize()
    want = []
    for _ in range(3):
        run()
        st.synchronize()
        want.append([t.clone() for t in results])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        run()
    for t in results:
        t.zero_()
    torch.cuda.synchronize()
    for w in want:
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results, w))
