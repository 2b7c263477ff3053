"""Adapters, head norms and clipping as they are used together, around the 8-bit projection: the example, other streams, CUDA graphs."""

import os
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

import paper_1811_10751_b200 as g            # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROFILED = any(k in os.environ for k in ("CUDA_INJECTION64_PATH", "NV_COMPUTE_PROFILER_PERFWORKS_DIR", "NV_NSIGHT_INJECTION_PORT_BASE"))


def _example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import adapter_step
    finally:
        sys.path.pop(0)
    return adapter_step


@pytest.mark.parametrize("args", [("300", "520", "16"), ("77", "256", "7")])
def test_example_is_as_near_to_fp32_as_its_roundings_allow(args):
    """The weights are the same on both sides; x is cut to e4m3 (2.6e-2 of each factor on average), so the projection is off by
    that much of its terms' root sum of squares, about the size of the result itself; BF16 roundings (2^-9 on average) vanish
    beside it.  Back through the norms: dx is projected out of the row's own direction, which keeps its size; d A and d B take
    their gradients from those.  e5m2 gradients (5.2e-2) enter d hidden.  Twice each figure bounds them."""
    T, H, r = args
    far = _example().main(["--tokens", T, "--hidden", H, "--rank", r])
    assert far["queries"] < 2 * 2.6e-2 and far["keys"] < 2 * 2.6e-2 and far["served queries"] < 2 * 2.6e-2 and far["served keys"] < 2 * 2.6e-2
    assert far["d A"] < 2 * 5.2e-2 and far["d B"] < 2 * 5.2e-2 and far["d hidden"] < 2 * 5.8e-2
    assert far["d query weight"] < 2 * 5.2e-2 and far["d key weight"] < 2 * 5.2e-2
    assert far["norm"] < 1e-6 and far["clipped"] < 1e-5


def _chain(T=130, H=264, r=24):
    ex = _example()
    gen = torch.Generator(device="cuda").manual_seed(5)
    rand = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    q_heads, k_heads, D, n = 4, 2, 64, 2
    N = (q_heads + k_heads) * D
    layer = ex.AdaptedHeads((rand(N, H) / 16).bfloat16(), (rand(n, r, H) / 16).bfloat16(), (rand(n, N, r) / 5).bfloat16(), torch.ones(n, device="cuda"),
                            torch.ones(D, device="cuda", dtype=torch.bfloat16), torch.ones(D, device="cuda", dtype=torch.bfloat16), q_heads, k_heads, D,
                            T, 512)
    x, pos = rand(T, H).bfloat16(), torch.randint(0, 512, (T,), device="cuda", generator=gen)
    dq, dk = rand(T, q_heads * D).bfloat16(), rand(T, k_heads * D).bfloat16()
    offsets, index = torch.tensor([0, 50, 51, 130], device="cuda"), torch.tensor([1, -1, 0], device="cuda")

    def run():
        layer.forward(x, pos, offsets, index)
        layer.backward(dq, dk, x, pos, offsets, index)
        layer.clip(0.5)
    outs = (layer.out, layer.h, layer.d, layer.dx, layer.dA, layer.dB, layer.dq_weight, layer.dk_weight, layer.norm)
    return run, outs


def test_chain_on_another_stream_and_replayed_from_a_graph_leaves_the_same_bits():
    run, outs = _chain()
    run()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    st = torch.cuda.Stream()
    for t in outs:
        t.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        run()
    st.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    if not PROFILED:                                   # ncu ends a process that launches into a stream capture
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            run()
        for _ in range(2):
            for t in outs:
                t.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs, want))
    assert g.gpd_device_status() == 0


def test_two_chains_at_once_with_workspaces_of_their_own():
    a, b = _chain(), _chain(T=130, H=520)
    for run, _ in (a, b):
        run()
    torch.cuda.synchronize()
    want = [[t.clone() for t in outs] for _, outs in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for (run, _), st in zip((a, b), streams):
            with torch.cuda.stream(st):
                run()
    torch.cuda.synchronize()
    for (_, outs), w in zip((a, b), want):
        assert all(torch.equal(x, y) for x, y in zip(outs, w))
