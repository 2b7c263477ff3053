"""The low-precision operators as they are used together: the example's whole step, other streams, CUDA graphs."""

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


def test_output_head_example_is_as_near_to_fp32_as_8_bits_allow():
    """e4m3 rounds each factor by at most 2^-4, on average (uniform in the mantissa) by 2.6e-2, so a product of two by
    3.7e-2 of its terms' root sum of squares; e5m2 gradients double their share (5.2e-2 with 2.6e-2: 5.8e-2).  The
    logits feed the log probabilities and the gradient, each with its own further rounding: twice the product's figure
    bounds all but the entropy and the norm's gradient, which average over many terms."""
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import output_head
    finally:
        sys.path.pop(0)
    far = output_head.main(["--tokens", "200", "--hidden", "520", "--vocab", "3001"])
    assert far["logits"] < 2 * 3.7e-2
    assert far["log probabilities"] < 2 * 3.7e-2 and far["entropy"] < 2 * 3.7e-2 and far["loss"] < 2 * 3.7e-2
    assert far["d hidden"] < 2 * 5.8e-2 and far["d weight"] < 2 * 5.8e-2 and far["d norm weight"] < 2 * 5.8e-2


def _chain(T=96, H=384, V=1000):
    gen = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    x, r, w = rand(T, H).bfloat16(), rand(T, H).bfloat16(), torch.ones(H, device="cuda", dtype=torch.bfloat16)
    W = rand(V, H).bfloat16() / 16
    q, s = g.new_fp8(T, H)
    wq, ws = g.new_fp8(V, H, block_rows=128)
    dq, ds = g.new_fp8(T, V, torch.float8_e5m2)
    wqT, wsT = g.new_fp8(H, V, block_rows=128)
    h, rstd = torch.empty_like(x), torch.empty(T, device="cuda")
    logits, d = torch.empty((T, V), device="cuda"), torch.empty((T, V), device="cuda")
    tok = torch.randint(0, V, (T,), device="cuda", generator=gen)
    lp, lse, H_ = (torch.empty(T, device="cuda") for _ in range(3))
    ids, tlp = torch.empty((T, 5), dtype=torch.int32, device="cuda"), torch.empty((T, 5), device="cuda")
    t_ids, t_log = torch.randint(0, V, (T, 7), device="cuda", generator=gen), rand(T, 7)
    loss, dl = torch.empty(T, device="cuda"), torch.empty((T, V), device="cuda")
    dy, dx, dw, wsp = torch.empty((T, H), device="cuda").bfloat16(), torch.empty_like(x), torch.empty(H, device="cuda"), torch.empty(T * H, device="cuda")

    def run(stream=None):
        g.gpd_quantize_blocks(W, q=wq, scales=ws, qT=wqT, scalesT=wsT, block_rows=128, stream=stream)
        g.gpd_rmsnorm_quant(x, w, 1e-5, residual=r, residual_out=h, q=q, scales=s, rstd=rstd, stream=stream)
        g.gpd_gemm_fp8(q, s, wq, ws, logits, stream=stream)
        g.gpd_token_logprobs(logits, tok, lp, lse, entropy=H_, top_ids=ids, top_logprobs=tlp, stream=stream)
        g.gpd_token_logprobs_backward(logits, tok, lse, H_, lp, lse, d, stream=stream)
        g.gpd_distill_topk(logits, t_ids, t_log, None, loss, dlogits=dl, stream=stream)
        g.gpd_quantize_blocks(dl, q=dq, scales=ds, stream=stream)
        g.gpd_gemm_fp8(dq, ds, wqT, wsT, dy, stream=stream)
        g.gpd_rmsnorm_backward(dy, h, w, rstd, dx, dw, wsp, stream=stream)
    return run, (q, s, h, rstd, logits, lp, lse, H_, ids, tlp, d, loss, dl, dy, dx, dw)


def _bytes(ts):
    return [t.contiguous().view(torch.uint8).clone() for t in ts]


def _spoil(ts):
    for t in ts:
        t.copy_(torch.zeros((), device="cuda").to(t.dtype).expand(t.shape))


def test_chain_on_another_stream_leaves_the_same_bits():
    run, outs = _chain()
    run()
    torch.cuda.synchronize()
    want = _bytes(outs)
    for way in ("argument", "handle", "current"):
        _spoil(outs)
        torch.cuda.synchronize()
        st = torch.cuda.Stream()
        if way == "current":
            with torch.cuda.stream(st):
                run()
        else:
            run(st if way == "argument" else st.cuda_stream)
        st.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(_bytes(outs), want)), way
    assert g.gpd_device_status() == 0


@pytest.mark.skipif(PROFILED, reason="a profiler is attached: ncu ends a process that launches into a stream capture")
def test_chain_replayed_from_a_cuda_graph_leaves_the_same_bits():
    run, outs = _chain()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        run(st)
    torch.cuda.synchronize()
    want = _bytes(outs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        run(st)
    for _ in range(2):
        _spoil(outs)
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(_bytes(outs), want))
    assert g.gpd_device_status() == 0
