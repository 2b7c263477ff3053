"""Tensors of more than 2^31 elements: offsets of rows do not fit in 32 bits.  The first and the last rows (and columns, where
the output is transposed) are held against 64-bit forms; bounds as in the tests of the single operators."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

import paper_1811_10751_b200 as g                                          # noqa: E402
from tests.lm_reference import check_close, check_cut, scale_values, spread   # noqa: E402

E4, E5, BF = torch.float8_e4m3fn, torch.float8_e5m2, torch.bfloat16
REL = 2e-5


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(seed, rows, cols):
    x = torch.empty((rows, cols), dtype=BF, device="cuda")
    for r in range(0, rows, 1 << 16):                        # randn makes FP32 numbers first
        n = min(1 << 16, rows - r)
        x[r:r + n] = torch.randn((n, cols), device="cuda", generator=_gen(seed + r))
    return x


def _ends(n, k=3):
    return torch.tensor([*range(k), *range(n - k, n)], device="cuda")


@pytest.fixture(autouse=True)
def free_memory():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def test_norm_and_its_gradient():
    T, H = 262144 + 300, 8200
    x, w = _normal(1, T, H), (1 + 0.1 * torch.randn(H, device="cuda", generator=_gen(2))).to(BF)
    y, rstd = torch.empty_like(x), torch.empty(T, device="cuda")
    q, s = g.new_fp8(T, H)
    assert x.numel() > 2 ** 31 and q.stride(0) * T > 2 ** 31
    g.gpd_rmsnorm_quant(x, w, 1e-5, y=y, q=q, scales=s, rstd=rstd)
    at = _ends(T)
    h, wd = x[at].double(), w.double()
    r = (h.square().mean(1) + 1e-5).rsqrt()
    check_close(rstd[at], r, 2.0 ** -18)
    ref = h * r[:, None] * wd
    check_close(y[at], ref, 2.0 ** -18)
    check_cut(q.view(torch.uint8)[at].view(E4), s.view(torch.uint8)[at], ref, 2.0 ** -18)
    dx, dw, ws = y, torch.empty(H, device="cuda"), torch.empty(g.GPD_RMSNORM_MAX_PARTS * H, device="cuda")
    g.gpd_rmsnorm_backward(x, x, w, rstd, dx, dw, ws)        # dy = h
    gr = h * wd
    ref = r[:, None] * (gr - h * (r[:, None] ** 2) * (gr * h).mean(1, keepdim=True))
    size = r[:, None] * (gr.abs() + h.abs() * (r[:, None] ** 2) * (gr * h).abs().mean(1, keepdim=True))
    check_close(dx[at], ref, 2.0 ** -16, size)
    total = torch.zeros(H, device="cuda", dtype=torch.float64)
    for i in range(0, T, 1 << 14):
        total += (x[i:i + (1 << 14)].double().square() * rstd[i:i + (1 << 14), None].double()).sum(0)
    # positive terms: chains of T / 148 additions in a thread, then 148 rows
    check_close(dw, total, (T / 148 + 160) * 2.0 ** -24)


def test_cut_both_ways():
    M, K = 262144 + 40, 8200
    x = _normal(1, M, K)
    q, s = g.new_fp8(M, K, E5)
    qT, sT = g.new_fp8(K, M, E5)
    g.gpd_quantize_blocks(x, q=q, scales=s, qT=qT, scalesT=sT)
    rows, cols = _ends(M), _ends(K)
    check_cut(q.view(torch.uint8)[rows].view(E5), s.view(torch.uint8)[rows], x[rows].double(), 0.0)
    first = (M - 1000) // 128 * 128                          # whole blocks along the columns
    part = x[first:][:, cols].t().double()
    check_cut(qT.view(torch.uint8)[cols][:, first:].view(E5), sT.view(torch.uint8)[cols][:, first // 128:], part, 0.0)


@pytest.mark.parametrize("out", [BF, torch.float32])
def test_product(out):
    M, N, K = 270000, 8200, 8200 if out == BF else 640
    A, sa = g.new_fp8(M, K)
    B, sb = g.new_fp8(N, K, block_rows=128)
    for r in range(0, M, 1 << 15):
        n = min(1 << 15, M - r)
        A[r:r + n] = torch.randn((n, K), device="cuda", generator=_gen(r)).to(E4)
    B.copy_(torch.randn((N, K), device="cuda", generator=_gen(7)).to(E4))
    sa.view(torch.uint8).copy_(torch.randint(125, 130, sa.shape, device="cuda", generator=_gen(8)))
    sb.view(torch.uint8).copy_(torch.randint(125, 130, sb.shape, device="cuda", generator=_gen(9)))
    D = torch.empty((M, N), dtype=out, device="cuda")
    assert D.numel() > 2 ** 31
    g.gpd_gemm_fp8(A, sa, B, sb, D)
    assert g.gpd_device_status() == 0
    at = _ends(M, 130)
    a = A.view(torch.uint8)[at].view(E4).double() * scale_values(sa.view(torch.uint8)[at]).repeat_interleave(128, 1)[:, :K]
    b = B.double() * spread(scale_values(sb), 128, N, K)
    n = (20 + K / 512) if out == torch.float32 else (K / 32 + 4)
    check_close(D[at], a @ b.t(), n * 2.0 ** -23, a.abs() @ b.abs().t())


def test_logits():
    T, V, K = 16800, 128003, 8
    x = _normal(1, T, V)
    x *= 2
    assert x.numel() > 2 ** 31
    tok = torch.randint(0, V, (T,), device="cuda", generator=_gen(2))
    lp, lse, H = (torch.empty(T, device="cuda") for _ in range(3))
    ids, tlp = torch.empty((T, K), device="cuda", dtype=torch.int32), torch.empty((T, K), device="cuda")
    g.gpd_token_logprobs(x, tok, lp, lse, entropy=H, top_ids=ids, top_logprobs=tlp)
    at = _ends(T)
    z = x[at].double()
    logp = torch.log_softmax(z, 1)
    p = logp.exp()
    Hd = -(p * logp).sum(1)
    assert bool(((lp[at].double() - logp.gather(1, tok[at][:, None])[:, 0]).abs() < 1e-4).all())
    assert bool(((H[at].double() - Hd).abs() < REL * 14).all())
    want = torch.sort(x[at].float().cpu(), dim=1, descending=True, stable=True).indices[:, :K]
    assert torch.equal(ids[at].long().cpu(), want)
    gl, gh = torch.randn(T, device="cuda", generator=_gen(3)), torch.randn(T, device="cuda", generator=_gen(4))
    d = torch.empty_like(x)
    g.gpd_token_logprobs_backward(x, tok, lse, H, gl, gh, d)
    one = torch.zeros_like(p).scatter_(1, tok[at][:, None], 1.0)
    a, b = gl[at].double()[:, None], gh[at].double()[:, None]
    ref = a * (one - p) - b * p * (logp + Hd[:, None])
    size = a.abs() * (one + p) + b.abs() * p * (z.abs() + lse[at].double()[:, None].abs() + Hd[:, None])
    check_close(d[at], ref, REL + 2.0 ** -20 * float(z.abs().max()), size)
    t_ids, t_log = torch.randint(0, V, (T, 20), device="cuda", dtype=torch.int32, generator=_gen(5)), torch.randn((T, 20), device="cuda", generator=_gen(6))
    loss = torch.empty(T, device="cuda")
    g.gpd_distill_topk(x, t_ids, t_log, None, loss, dlogits=d)
    logq = torch.log_softmax(t_log[at].double(), 1)
    q, where = logq.exp(), t_ids[at].long()
    assert bool(((loss[at].double() - (q * (logq - logp.gather(1, where))).sum(1)).abs() < REL * 60).all())
    spot = torch.zeros_like(p).scatter_add_(1, where, q)
    check_close(d[at], p - spot, REL + 2.0 ** -20 * float(z.abs().max()), p + spot)
