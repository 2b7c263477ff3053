"""Log probabilities, entropy, top alternatives, their gradient, and distillation from top logits, against 64 bits.

Bounds.  One 2^x is off by at most 2^-22 (its argument, up to 40 in size where it matters, by 40 * 2^-23); a sum
has chains of at most 1100 terms in a thread and 30 merges: relative error below 8e-5 in the worst case and, with
roundings of either sign, below 1e-5; REL = 2e-5 is used for sums, probabilities and, absolutely, for logarithms of
sums and for the entropy (whose terms p log p it multiplies by at most 1 + H).  z = x / tau adds 2^-22 |z|."""

import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

import paper_1811_10751_b200 as g                            # noqa: E402
from tests.lm_reference import check_close, like, strided    # noqa: E402

BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32
REL = 2e-5
NAN, INF = float("nan"), float("inf")


def _rand(seed, *shape):
    return torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


def _ints(seed, hi, *shape):
    return torch.randint(0, hi, shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


def _top(logits, K):
    """Indices by value, then by index, NaN first (on the CPU, a stable sort)."""
    x = logits.float().cpu()
    return torch.sort(x + 0.0, dim=1, descending=True, stable=True).indices[:, :K]


def _near(got, ref, bound):
    assert torch.equal(torch.isnan(got), torch.isnan(ref)) and torch.equal(torch.isinf(got), torch.isinf(ref))
    ok = torch.isfinite(ref)
    assert bool(((got.double() - ref).abs() <= bound)[ok].all()), float(((got.double() - ref).abs() / bound)[ok].max())


SHAPES = [(1, 1, 0, 0), (3, 5, 0, 0), (2, 33, 1, 1), (5, 1000, 0, 3), (1, 1025, 7, 0), (7, 4099, 0, 1), (1, 16384, 0, 0),
          (2, 50257, 0, 0), (16, 32000, 0, 0), (3, 131075, 5, 2), (200, 9001, 0, 0), (1, 262144, 0, 0)]


@pytest.mark.parametrize("T,V,pad,offset", SHAPES)
@pytest.mark.parametrize("dtype,index,G,K,tau", [(BF, torch.int32, 1, 0, 1.0), (HF, torch.int64, 3, 5, 0.7), (F32, torch.int32, 1, 20, 1.3),
                                                 (BF, torch.int64, 64, 32, 0.5)])
def test_logprobs_match_64_bit_form(T, V, pad, offset, dtype, index, G, K, tau):
    K = min(K, V)
    x = like(_rand(1, T, V) * 3, dtype, pad, offset)
    tok = _ints(2, V, T, G).to(index)
    if G > 1:
        tok[0, 1], tok[0, 2 % G] = -1, tok[0, 0]
    lp, lse, H = torch.empty((T, G), device="cuda"), torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    ids = torch.empty((T, K), device="cuda", dtype=torch.int32) if K else None
    tlp = torch.empty((T, K), device="cuda") if K else None
    g.gpd_token_logprobs(x, tok[:, 0].contiguous() if G == 1 else tok, lp[:, 0] if G == 1 else lp, lse, entropy=H, top_ids=ids,
                         top_logprobs=tlp, temperature=tau)
    z = x.double() / tau
    rl = torch.logsumexp(z, 1)
    logp = z - rl[:, None]
    zmax = z.abs().amax(1)
    _near(lse, rl, REL + 2.0 ** -22 * zmax)
    _near(H, -(logp.exp() * logp).sum(1), REL * (2 + math.log(V)))
    ref = torch.where(tok >= 0, logp.gather(1, tok.clamp(min=0).long()), 0.0)
    _near(lp, ref, (REL + 2.0 ** -20 * zmax)[:, None])
    if K:
        want = _top(x, K)
        assert torch.equal(ids.long().cpu(), want)
        _near(tlp, logp.gather(1, want.cuda()), (REL + 2.0 ** -20 * zmax)[:, None])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [40, 5000, 70001])
def test_top_alternatives_with_ties_masks_and_special_values(V, dtype):
    T, K = 8, 32
    x = _rand(1, T, V).to(dtype)
    x[0] = 1.5                                                   # all equal
    x[1] = -INF                                                  # nothing left
    x[2, :] = -INF
    x[2, V - 3:] = 2.0                                           # fewer than K left
    x[3] = torch.finfo(dtype).min                                # a mask of the lowest value, everywhere
    x[4, :] = torch.finfo(dtype).min
    x[4, 7] = -3.0                                               # and everywhere but in one place
    x[5, V // 2] = NAN
    x[6, 5] = INF
    x[7] = (x[7] * 2).round() / 2                                # many equal values, two zeros
    tok = torch.tensor([0, 1, V - 1, 3, 7, 1, 5, V], device="cuda")
    lp, lse, H = (torch.empty(T, device="cuda") for _ in range(3))
    ids, tlp = torch.empty((T, K), device="cuda", dtype=torch.int32), torch.empty((T, K), device="cuda")
    g.gpd_token_logprobs(x, tok, lp, lse, entropy=H, top_ids=ids, top_logprobs=tlp)
    assert torch.equal(ids.long().cpu(), _top(x, K))
    lnV = math.log(V)
    assert abs(float(lp[0]) + lnV) < REL * 12 and abs(float(H[0]) - lnV) < REL * 12
    assert float(lse[1]) == -INF and float(lp[1]) == -INF and float(H[1]) == 0 and bool((tlp[1] == -INF).all())
    assert abs(float(lp[2]) + math.log(3)) < REL and abs(float(H[2]) - math.log(3)) < REL
    assert abs(float(H[3]) - lnV) < REL * 12                      # all equal again
    assert abs(float(lp[4])) < REL and abs(float(H[4])) < REL
    for r in (5, 6):
        assert all(math.isnan(float(v[r])) for v in (lp, lse, H))
    assert math.isnan(float(lp[7])) and math.isfinite(float(lse[7]))   # a token beyond the row
    none = torch.empty((0, V), device="cuda", dtype=dtype)
    e = torch.empty(0, device="cuda")
    g.gpd_token_logprobs(none, torch.empty(0, device="cuda", dtype=torch.int32), e, e)


@pytest.mark.parametrize("T,V,pad,offset", SHAPES)
@pytest.mark.parametrize("dtype,G,tau,which", [(BF, 1, 1.0, "both"), (F32, 3, 0.7, "both"), (HF, 64, 1.5, "tokens"), (F32, 1, 1.0, "entropy")])
def test_logprobs_gradient_matches_64_bit_form(T, V, pad, offset, dtype, G, tau, which):
    x = like(_rand(1, T, V) * 3, dtype, pad, offset)
    tok = _ints(2, V, T, G)
    if G > 1:
        tok[0, 1], tok[0, 2 % G] = -1, tok[0, 0]
    z = x.double() / tau
    lse = torch.logsumexp(z, 1)
    logp = z - lse[:, None]
    p = logp.exp()
    H = -(p * logp).sum(1)
    gl = _rand(3, T, G) if which != "entropy" else None
    gh = _rand(4, T) if which != "tokens" else None
    d = strided(T, V, dtype, pad + 3, offset + 1)
    g.gpd_token_logprobs_backward(x, tok if G > 1 else tok[:, 0].contiguous(), lse.float(), H.float(), gl, gh, d, temperature=tau)
    a = torch.zeros((T, G), device="cuda", dtype=torch.float64) if gl is None else torch.where(tok >= 0, gl.double(), 0.0)
    b = torch.zeros(T, device="cuda", dtype=torch.float64) if gh is None else gh.double()
    one = torch.zeros((T, V), device="cuda", dtype=torch.float64).scatter_add_(1, tok.clamp(min=0), a)
    abs1 = torch.zeros((T, V), device="cuda", dtype=torch.float64).scatter_add_(1, tok.clamp(min=0), a.abs())
    ref = (one - p * a.sum(1, keepdim=True) - b[:, None] * p * (logp + H[:, None])) / tau
    # z - lse is a difference of FP32 numbers: its error goes by their size, not by its own
    size = (abs1 + p * a.abs().sum(1, keepdim=True) + b.abs()[:, None] * p * (z.abs() + lse.abs()[:, None] + H[:, None])) / tau
    check_close(d, ref, REL + 2.0 ** -20 * float(z.abs().max()), size)
    d2 = like(x, dtype, pad, offset)
    g.gpd_token_logprobs_backward(d2, tok if G > 1 else tok[:, 0].contiguous(), lse.float(), H.float(), gl, gh, d2, temperature=tau)
    assert torch.equal(d2, d)                                    # over the logits themselves


def test_logprobs_gradient_against_differences_and_of_masked_rows():
    T, V, G, tau = 3, 700, 2, 0.8
    x, tok, gl, gh = _rand(1, T, V), _ints(2, V, T, G), _rand(3, T, G), _rand(4, T)

    def value(x):
        logp = torch.log_softmax(x / tau, 1)
        return (logp.gather(1, tok) * gl.double()).sum() - (gh.double() * (logp.exp() * logp).sum(1)).sum()
    lp, lse, H = torch.empty((T, G), device="cuda"), torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    g.gpd_token_logprobs(x, tok, lp, lse, entropy=H, temperature=tau)
    d = torch.empty_like(x)
    g.gpd_token_logprobs_backward(x, tok, lse, H, gl, gh, d, temperature=tau)
    for s in range(4):
        v, e = _rand(10 + s, T, V).double(), 1e-4
        num = (value(x.double() + e * v) - value(x.double() - e * v)) / (2 * e)
        assert abs(float((d.double() * v).sum() - num)) <= 1e-5 * float((d.double() * v).abs().sum())
    x = _rand(5, 4, 600)
    x[0], x[1, ::2], x[2, 3] = -INF, -INF, NAN
    tok = torch.tensor([5, 1, 2, 9], device="cuda", dtype=torch.int32)
    tok[3] = 600                                                 # beyond the row: no gradient
    lp, lse, H = (torch.empty(4, device="cuda") for _ in range(3))
    g.gpd_token_logprobs(x, tok, lp, lse, entropy=H)
    d = torch.full_like(x, 7.0)
    g.gpd_token_logprobs_backward(x, tok, lse, H, torch.ones(4, device="cuda"), torch.ones(4, device="cuda"), d)
    assert bool((d[0] == 0).all()) and bool(torch.isfinite(d[1]).all()) and bool((d[1, ::2] == 0).all())
    assert bool(torch.isnan(d[2]).all())
    logp = torch.log_softmax(x[3].double(), 0)
    check_close(d[3:4], (-logp.exp() * (logp + H[3].double()))[None], 1e-4, logp.exp()[None] * 10)


def _distill_ref(x, ids, t, w, tau):
    logp = torch.log_softmax(x.double() / tau, 1)
    ok = ids >= 0
    logq = torch.log_softmax((t.double() / tau).masked_fill(~ok, -INF), 1)
    q = logq.exp()
    loss = (torch.where(q > 0, q * (logq - logp.gather(1, ids.clamp(min=0).long())), 0.0)).sum(1) * w * tau * tau
    s = torch.zeros_like(logp).scatter_add_(1, ids.clamp(min=0).long(), q)
    return loss, (logp.exp() - s) * (w * tau)[:, None], (logp.exp() + s) * (w * tau).abs()[:, None]


@pytest.mark.parametrize("T,V,pad,offset", SHAPES)
@pytest.mark.parametrize("dtype,ttype,index,K,tau", [(BF, F32, torch.int32, 1, 1.0), (F32, BF, torch.int64, 20, 2.0), (HF, HF, torch.int32, 64, 0.7),
                                                     (F32, F32, torch.int32, 1000, 1.0)])
def test_distillation_matches_64_bit_form(T, V, pad, offset, dtype, ttype, index, K, tau):
    x = like(_rand(1, T, V) * 3, dtype, pad, offset)
    ids = like(_ints(2, V, T, K), index, pad, 0)                  # duplicates among them
    t = like(_rand(3, T, K) * 2, ttype, pad, 1)
    if K > 1:
        ids[0, K // 2:] = -1                                      # a shorter list
        t[T - 1, 0] = -INF
    w = _rand(4, T)
    if T > 2:
        w[1] = 0
    loss, d = torch.full((T,), NAN, device="cuda"), strided(T, V, dtype, pad + 3, offset + 1)
    g.gpd_distill_topk(x, ids, t, w, loss, dlogits=d, temperature=tau)
    rl, rd, size = _distill_ref(x, ids, t, w.double(), tau)
    zmax = float(x.double().abs().max()) / tau
    # the terms of the loss are of either sign: bounded by their sizes
    bound = w.double().abs() * tau * tau * (REL * 3 + 2.0 ** -20 * (zmax + float(t[torch.isfinite(t)].double().abs().max()) / tau)) * (2 + 2 * zmax)
    _near(loss, rl, bound)
    check_close(d, rd, REL + 2.0 ** -20 * zmax, size)
    loss2 = torch.empty_like(loss)
    g.gpd_distill_topk(x, ids, t, w, loss2, temperature=tau)      # the loss alone
    assert torch.equal(loss, loss2)
    d2 = like(x, dtype, pad, offset)                              # the same alignment, so the same order of sums
    g.gpd_distill_topk(d2, ids, t, w, loss2, dlogits=d2, temperature=tau)
    assert torch.equal(d2, d) and torch.equal(loss, loss2)        # over the logits themselves


def test_distillation_gradient_against_differences():
    T, V, K, tau = 3, 900, 7, 1.7
    x, ids, t, w = _rand(1, T, V), _ints(2, V, T, K), _rand(3, T, K), _rand(4, T)
    loss, d = torch.empty(T, device="cuda"), torch.empty_like(x)
    g.gpd_distill_topk(x, ids, t, w, loss, dlogits=d, temperature=tau)
    for s in range(4):
        v, e = _rand(10 + s, T, V).double(), 1e-4
        num = (_distill_ref(x.double() + e * v, ids, t, w.double(), tau)[0] - _distill_ref(x.double() - e * v, ids, t, w.double(), tau)[0]).sum() / (2 * e)
        assert abs(float((d.double() * v).sum() - num)) <= 1e-5 * float((d.double() * v).abs().sum())


@pytest.mark.parametrize("V", [500, 60000])
def test_distillation_of_rows_without_weight_list_or_logits(V):
    T, K = 7, 4
    x, t = _rand(1, T, V), _rand(2, T, K)
    ids = _ints(3, V, T, K)
    w = torch.ones(T, device="cuda")
    x[0], w[0] = NAN, 0.0                                         # no weight: not read
    ids[1] = -1                                                   # an empty list
    t[2] = -INF
    x[3] = -INF                                                   # no logits
    ids[4, 2] = V                                                 # beyond the row
    x[5, 9] = -INF
    ids[5] = torch.tensor([9, 10, 11, 12])                        # a masked entry that the teacher wants
    t[6, 1] = NAN
    loss, d = torch.full((T,), 5.0, device="cuda"), torch.full_like(x, 5.0)
    g.gpd_distill_topk(x, ids, t, w, loss, dlogits=d)
    assert [float(v) for v in loss[:4]] == [0.0, 0.0, 0.0, INF]
    assert all(bool((d[r] == 0).all()) for r in range(4))
    assert math.isnan(float(loss[4])) and float(loss[5]) == INF and math.isnan(float(loss[6]))
    q = torch.softmax(t[5].double(), 0)
    p = torch.softmax(x[5].double(), 0)
    p[9:13] -= q
    check_close(d[5:6], p[None], REL * 2, p.abs()[None] + 1e-3)
    e, ei = torch.empty((0, V), device="cuda"), torch.empty((0, K), device="cuda", dtype=torch.int32)
    g.gpd_distill_topk(e, ei, ei.float(), None, torch.empty(0, device="cuda"))
    k0 = torch.empty((T, 0), device="cuda", dtype=torch.int32)    # lists of no entries
    g.gpd_distill_topk(x, k0, k0.float(), None, loss, dlogits=d)
    assert bool((loss == 0).all()) and bool((d == 0).all())


def test_refusals():
    T, V = 4, 64
    x, tok = torch.zeros((T, V), device="cuda"), torch.zeros(T, device="cuda", dtype=torch.int32)
    f, ids = torch.empty(T, device="cuda"), torch.empty((T, 3), device="cuda", dtype=torch.int32)
    for kw in (dict(tokens=tok.float()), dict(lse=f[:3]), dict(lse=None), dict(top_logprobs=ids.float()), dict(top_ids=ids.long()),
               dict(tokens=tok[None]), dict(logits=x.double()), dict(logits=x.cpu()), dict(entropy=f.double())):
        args = dict(logits=x, tokens=tok, logprobs=f, lse=f.clone())
        args.update(kw)
        with pytest.raises(ValueError):
            g.gpd_token_logprobs(**args)
    for kw, status in ((dict(temperature=0.0), g.GPD_ERR_ARG), (dict(temperature=-1.0), g.GPD_ERR_ARG), (dict(temperature=NAN), g.GPD_ERR_ARG),
                       (dict(temperature=INF), g.GPD_ERR_ARG), (dict(top_ids=torch.empty((T, 33), device="cuda", dtype=torch.int32)), g.GPD_ERR_SHAPE),
                       (dict(tokens=tok[:, None].expand(T, 65).contiguous(), logprobs=torch.empty((T, 65), device="cuda")), g.GPD_ERR_SHAPE)):
        args = dict(logits=x, tokens=tok, logprobs=f, lse=f.clone())
        args.update(kw)
        with pytest.raises(g.GpdError) as e:
            g.gpd_token_logprobs(**args)
        assert e.value.status == status
    with pytest.raises(g.GpdError) as e:                          # more alternatives than entries
        g.gpd_token_logprobs(x[:, :2], tok, f, f.clone(), top_ids=ids)
    assert e.value.status == g.GPD_ERR_SHAPE
    with pytest.raises(g.GpdError) as e:                          # entropy's gradient without the entropy
        g.gpd_token_logprobs_backward(x, tok, f, None, None, f, x.clone())
    assert e.value.status == g.GPD_ERR_ARG
    with pytest.raises(ValueError):
        g.gpd_token_logprobs_backward(x, tok, f, None, f, None, x.clone().half())
    for a in ((x, ids, x[:, :2], None, f), (x, ids.float(), ids.float(), None, f), (x, ids, ids.float(), f[:2], f), (x, ids, ids.float(), None, f[:2])):
        with pytest.raises(ValueError):
            g.gpd_distill_topk(*a)
    with pytest.raises(g.GpdError) as e:
        big = torch.zeros((T, 1025), device="cuda")
        g.gpd_distill_topk(x, big.int(), big, None, f)
    assert e.value.status == g.GPD_ERR_SHAPE
    with pytest.raises(g.GpdError):
        g.gpd_distill_topk(x, ids, ids.float(), None, f, temperature=0.0)
