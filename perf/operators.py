"""Cases, plain forms and calls of the low-precision layer and output-head operators.

The operators are those around the last layers of a language model: the root-mean-square norm with the
residual's addition and an 8-bit output, the cutting of a matrix into 8-bit blocks, the 8-bit matrix
product with a scale for each block of 128, the log probabilities of given tokens, and distillation from
a teacher's top logits.

8-bit values are e4m3 or e5m2 numbers; 128 neighbours along the contraction share one power-of-two
scale, the smallest with which the largest of them stays within the type's range, held as an 8-bit
exponent (e8m0).  A block without a non-zero value has the scale 1.

`run` with `own` false computes the operators from elementary torch operations in 32 bits, rounded once;
with `own` true it makes the calls of the framework.  `exact` gives the same outputs from the definitions
in 64 bits (8-bit outputs before their rounding, which both sides share).
"""

import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16,
          "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
_TOP = {"e4m3": 448.0, "e5m2": 57344.0}
_E8M0 = torch.float8_e8m0fnu
_EPS = 1e-5


# ---- cases ----------------------------------------------------------------------------------------
def listed():
    return [
        # the norm in front of a layer while a handful of sequences produce one token each: latency
        dict(name="norm decode", op="norm", T=4, H=4096, type="bf16", q="e4m3", train=False),
        # the same norm over a long batch of prompts
        dict(name="norm prompts", op="norm", T=8192, H=8192, type="bf16", q="e4m3", train=True),
        # its backward pass in a training step of a middle-sized layer
        dict(name="norm backward", op="norm_bwd", T=4096, H=4096, type="bf16"),
        # output gradients cut for both of the products that follow (rows for dX, columns for dW)
        dict(name="cut gradients", op="cut", M=4096, K=8192, type="bf16", q="e5m2", block_rows=1, both=True),
        # FP32 master weights cut into 128 x 128 blocks after an optimizer step, odd row count
        dict(name="cut weights", op="cut", M=1000, K=4096, type="f32", q="e4m3", block_rows=128, both=True),
        # one projection while seven sequences produce one token each: reads the weights, little else
        dict(name="product decode", op="product", M=7, N=4096, K=4096, a="e4m3", b="e4m3", b_rows=128, out="bf16"),
        # a projection of a full training batch
        dict(name="product forward", op="product", M=8192, N=8192, K=8192, a="e4m3", b="e4m3", b_rows=128, out="bf16"),
        # its weight gradient over a ragged number of tokens, scales along the tokens on both sides, FP32 result
        dict(name="product weight gradient", op="product", M=4096, N=4096, K=4100, a="e5m2", b="e4m3", b_rows=1, out="f32"),
        # sampling step of sixteen sequences: log probability, entropy and twenty alternatives
        dict(name="logprobs decode", op="logprobs", T=16, V=128000, type="f32", top=20, temperature=0.7),
        # policy-gradient step over an odd vocabulary: forward and backward
        dict(name="logprobs training", op="logprobs_bwd", T=2048, V=50257, type="bf16", temperature=1.0),
        # evaluation of a student on a short text against the teacher's top 20: loss alone
        dict(name="distill evaluation", op="distill", T=61, V=32000, type="bf16", K=20, temperature=1.0, grad=False),
        # distillation step: loss and gradient, the teacher's top 64, soft temperature
        dict(name="distill training", op="distill", T=4096, V=128000, type="bf16", K=64, temperature=2.0, grad=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_bwd", "cut", "product", "product", "product", "logprobs",
                     "logprobs_bwd", "distill", "distill"])
    t = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op in ("norm", "norm_bwd"):
        H = _log(rng, 64, 16384)
        T = _log(rng, 1, min(8192, 8192 * 8192 // H))
        if op == "norm":
            return dict(op=op, T=T, H=H, type=t, q=rng.choice(["e4m3", "e4m3", "e5m2"]), train=rng.random() < 0.5)
        return dict(op=op, T=T, H=H, type=t)
    if op == "cut":
        K = _log(rng, 64, 16384)
        M = _log(rng, 1, min(8192, 4096 * 8192 // K))
        return dict(op=op, M=M, K=K, type=t, q=rng.choice(["e4m3", "e5m2"]), block_rows=rng.choice([1, 128]),
                    both=rng.random() < 0.7)
    if op == "product":
        M, N, K = _log(rng, 1, 8192), _log(rng, 64, 8192), _log(rng, 64, 8192)
        return dict(op=op, M=M, N=N, K=K, a=rng.choice(["e4m3", "e4m3", "e5m2"]), b="e4m3",
                    b_rows=rng.choice([1, 128, 128]), out=rng.choice(["bf16", "bf16", "f16", "f32"]))
    V = _log(rng, 1000, 150000)
    T = _log(rng, 1, min(4096, 4096 * 64000 // V))
    tau = round(rng.uniform(0.6, 2.0), 2)
    if op == "logprobs":
        return dict(op=op, T=T, V=V, type=t, top=rng.choice([0, 1, 5, 20, 32]), temperature=tau)
    if op == "logprobs_bwd":
        return dict(op=op, T=T, V=V, type=t, temperature=tau)
    return dict(op=op, T=T, V=V, type=t, K=rng.choice([1, 8, 20, 64, 128]), temperature=tau, grad=rng.random() < 0.7)


# ---- inputs ---------------------------------------------------------------------------------------
def _padded(rows, cols, dtype, step):
    """[rows, cols] buffer whose rows start at multiples of `step` elements."""
    return torch.empty((rows, (cols + step - 1) // step * step), dtype=dtype, device="cuda")[:, :cols]


def _q_buffer(rows, cols, name):
    return _padded(rows, cols, _TYPES[name], 16)


def _scale_buffer(rows, cols):
    return _padded(rows, (cols + 127) // 128, _E8M0, 4)


def _operand(gen, rows, cols, name, block_rows):
    """8-bit operand with its scales: activations or gradients with a few loud columns, cut block by block."""
    x = torch.randn((rows, cols), device="cuda", generator=gen)
    x *= torch.exp(torch.randn((1, cols), device="cuda", generator=gen) * 0.7)
    q, s = _cut_plain(x, name, block_rows)
    qb, sb = _q_buffer(rows, cols, name), _scale_buffer(s.shape[0], cols)
    qb.copy_(q)
    sb.copy_(s)
    return qb, sb


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    rand = lambda *shape: torch.randn(shape, device="cuda", generator=gen)  # noqa: E731
    op, s = c["op"], {"case": c}
    if op in ("norm", "norm_bwd"):
        T, H, dt = c["T"], c["H"], _TYPES[c["type"]]
        spread = torch.exp(rand(1, H) * 0.5)                       # some channels are louder than others
        s["weight"] = (1.0 + 0.1 * rand(H)).to(dt)
        if op == "norm":
            s["x"], s["residual"] = (0.3 * rand(T, H)).to(dt), (rand(T, H) * spread).to(dt)
            s["residual_out"] = torch.empty_like(s["x"])
            s["q"], s["scales"] = _q_buffer(T, H, c["q"]), _scale_buffer(T, H)
            s["rstd"] = torch.empty(T, device="cuda")
        else:
            s["h"] = (rand(T, H) * spread).to(dt)
            s["rstd"] = torch.rsqrt(s["h"].float().square().mean(1) + _EPS)
            s["dy"], s["dresidual"] = (1e-2 * rand(T, H)).to(dt), (1e-2 * rand(T, H)).to(dt)
            s["dx"], s["dweight"] = torch.empty_like(s["h"]), torch.empty(H, device="cuda")
            s["workspace"] = torch.empty(512 * max(H, 1), device="cuda")   # one FP32 row for each of 512 partial sums
    elif op == "cut":
        M, K, dt, b = c["M"], c["K"], _TYPES[c["type"]], c["block_rows"]
        s["src"] = (rand(M, K) * torch.exp(rand(1, K) * 0.7)).to(dt)
        s["q"], s["scales"] = _q_buffer(M, K, c["q"]), _scale_buffer((M + b - 1) // b, K)
        if c["both"]:
            s["qT"], s["scalesT"] = _q_buffer(K, M, c["q"]), _scale_buffer((K + b - 1) // b, M)
    elif op == "product":
        s["A"], s["a_scales"] = _operand(gen, c["M"], c["K"], c["a"], 1)
        s["B"], s["b_scales"] = _operand(gen, c["N"], c["K"], c["b"], c["b_rows"])
        s["out"] = torch.empty((c["M"], c["N"]), dtype=_TYPES[c["out"]], device="cuda")
    else:
        T, V, dt = c["T"], c["V"], _TYPES[c["type"]]
        z = rand(T, V) * 2.5
        if op == "distill":
            K = c["K"]
            # the teacher sees much the same text: its logits follow the student's, with some of its own
            teacher = z * 0.8 + rand(T, V) * 1.5
            top = torch.topk(teacher, K, dim=1)
            del teacher
            ids, s["teacher_logits"] = top.indices.to(torch.int32), top.values.contiguous()
            short = torch.rand((T, 1), device="cuda", generator=gen) < 0.1     # some lists are shorter than K
            s["teacher_ids"] = torch.where(short & (torch.arange(K, device="cuda") >= (K + 1) // 2), -1, ids).contiguous()
            # rows of the prompt and of padding carry no weight
            s["weights"] = (torch.rand(T, device="cuda", generator=gen) >= 0.05).float() / T
            s["loss"] = torch.empty(T, device="cuda")
        else:
            s["tokens"] = torch.randint(0, V, (T,), device="cuda", generator=gen, dtype=torch.int32)
            z.scatter_add_(1, s["tokens"].long()[:, None], torch.full((T, 1), 6.0, device="cuda"))
            s["logprobs"], s["lse"], s["entropy"] = (torch.empty(T, device="cuda") for _ in range(3))
            if op == "logprobs":
                if c["top"]:
                    s["top_ids"] = torch.empty((T, c["top"]), device="cuda", dtype=torch.int32)
                    s["top_logprobs"] = torch.empty((T, c["top"]), device="cuda")
            else:
                s["dlogprobs"], s["dentropy"] = rand(T) / T, rand(T) * 0.01 / T
        s["logits"] = z.to(dt)
        if op == "logprobs_bwd" or c.get("grad"):
            s["dlogits"] = torch.empty_like(s["logits"])
    return s


# ---- one pass -------------------------------------------------------------------------------------
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    import paper_1811_10751_b200 as g
    c = s["case"]
    op = c["op"]
    if op == "norm":
        rstd = s["rstd"] if c["train"] else None
        g.gpd_rmsnorm_quant(s["x"], s["weight"], _EPS, residual=s["residual"], residual_out=s["residual_out"],
                            q=s["q"], scales=s["scales"], rstd=rstd)
        return {"residual": s["residual_out"], "q": s["q"], "scales": s["scales"], "rstd": rstd}
    if op == "norm_bwd":
        g.gpd_rmsnorm_backward(s["dy"], s["h"], s["weight"], s["rstd"], s["dx"], s["dweight"], s["workspace"],
                               dresidual=s["dresidual"])
        return {"dx": s["dx"], "dweight": s["dweight"]}
    if op == "cut":
        g.gpd_quantize_blocks(s["src"], q=s["q"], scales=s["scales"], qT=s.get("qT"), scalesT=s.get("scalesT"),
                              block_rows=c["block_rows"])
        return {k: s.get(k) for k in ("q", "scales", "qT", "scalesT")}
    if op == "product":
        g.gpd_gemm_fp8(s["A"], s["a_scales"], s["B"], s["b_scales"], s["out"])
        return s["out"]
    if op == "logprobs":
        g.gpd_token_logprobs(s["logits"], s["tokens"], s["logprobs"], s["lse"], entropy=s["entropy"],
                             top_ids=s.get("top_ids"), top_logprobs=s.get("top_logprobs"), temperature=c["temperature"])
        return {k: s.get(k) for k in ("logprobs", "lse", "entropy", "top_ids", "top_logprobs")}
    if op == "logprobs_bwd":
        g.gpd_token_logprobs(s["logits"], s["tokens"], s["logprobs"], s["lse"], entropy=s["entropy"],
                             temperature=c["temperature"])
        g.gpd_token_logprobs_backward(s["logits"], s["tokens"], s["lse"], s["entropy"], s["dlogprobs"], s["dentropy"],
                                      s["dlogits"], temperature=c["temperature"])
        return {k: s[k] for k in ("logprobs", "lse", "entropy", "dlogits")}
    g.gpd_distill_topk(s["logits"], s["teacher_ids"], s["teacher_logits"], s["weights"], s["loss"],
                       dlogits=s.get("dlogits"), temperature=c["temperature"])
    return {"loss": s["loss"], "dlogits": s.get("dlogits")}


def _block_max(x, block_rows):
    """Largest magnitude of each block of block_rows x 128."""
    rows, cols = x.shape
    rb, kb = (rows + block_rows - 1) // block_rows, (cols + 127) // 128
    a = torch.nn.functional.pad(x.abs(), (0, kb * 128 - cols, 0, rb * block_rows - rows))
    return a.view(rb, block_rows, kb, 128).amax(dim=(1, 3))


def _spread(s, block_rows, rows, cols):
    """A value for each element from a value for each block."""
    return s.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(128, 1)[:, :cols]


def _scale_exponent(amax, name):
    """Smallest e with amax <= top 2^e, from the binary exponent: top is 0.875 times a power of two."""
    m, e = torch.frexp(amax)
    e = e - int(math.log2(_TOP[name] / 0.875)) + (m > 0.875)
    return torch.where(amax > 0, e, torch.zeros_like(e))


def _cut_plain(x, name, block_rows):
    scale = torch.exp2(_scale_exponent(_block_max(x, block_rows), name).to(x.dtype))
    q = (x / _spread(scale, block_rows, *x.shape)).to(_TYPES[name])
    return q, scale.to(_E8M0)


def _run_plain(s):
    c = s["case"]
    op = c["op"]
    if op == "norm":
        h = s["x"].float() + s["residual"].float()
        rstd = torch.rsqrt(h.square().mean(1) + _EPS)
        q, scales = _cut_plain(h * rstd[:, None] * s["weight"].float(), c["q"], 1)
        return {"residual": h.to(s["x"].dtype), "q": q, "scales": scales, "rstd": rstd if c["train"] else None}
    if op == "norm_bwd":
        h, dy, r = s["h"].float(), s["dy"].float(), s["rstd"][:, None]
        gr = dy * s["weight"].float()
        dx = r * (gr - h * (r * r) * (gr * h).mean(1, keepdim=True)) + s["dresidual"].float()
        return {"dx": dx.to(s["h"].dtype), "dweight": (dy * h * r).sum(0)}
    if op == "cut":
        x = s["src"].float()
        q, scales = _cut_plain(x, c["q"], c["block_rows"])
        qT, scalesT = _cut_plain(x.t().contiguous(), c["q"], c["block_rows"]) if c["both"] else (None, None)
        return {"q": q, "scales": scales, "qT": qT, "scalesT": scalesT}
    if op == "product":
        A = s["A"].float() * _spread(s["a_scales"].float(), 1, *s["A"].shape)
        B = s["B"].float() * _spread(s["b_scales"].float(), c["b_rows"], *s["B"].shape)
        return (A @ B.t()).to(s["out"].dtype)
    z = s["logits"].float() / c["temperature"]
    m = z.amax(1, keepdim=True)
    if op in ("logprobs", "logprobs_bwd"):
        e = torch.exp(z - m)
        S = e.sum(1, keepdim=True)
        lse = m + torch.log(S)
        H = torch.log(S[:, 0]) - (e * (z - m)).sum(1) / S[:, 0]
        at = s["tokens"].long()[:, None]
        out = {"logprobs": (z.gather(1, at) - lse)[:, 0], "lse": lse[:, 0], "entropy": H}
        if op == "logprobs":
            ids = _top_plain(s["logits"], c["top"]) if c["top"] else None
            out["top_ids"] = ids.to(torch.int32) if c["top"] else None
            out["top_logprobs"] = z.gather(1, ids) - lse if c["top"] else None
            return out
        p, logp = e / S, z - lse
        gl, gh = s["dlogprobs"][:, None], s["dentropy"][:, None]
        d = -gl * p - gh * p * (logp + H[:, None])
        d.scatter_add_(1, at, gl)
        out["dlogits"] = (d / c["temperature"]).to(s["logits"].dtype)
        return out
    tau, w = c["temperature"], s["weights"]
    valid = s["teacher_ids"] >= 0
    at = torch.where(valid, s["teacher_ids"], 0).long()
    t = torch.where(valid, s["teacher_logits"] / tau, -math.inf)
    te = torch.exp(t - t.amax(1, keepdim=True))
    q = te / te.sum(1, keepdim=True)
    e = torch.exp(z - m)
    S = e.sum(1, keepdim=True)
    logp = z.gather(1, at) - m - torch.log(S)
    logq = torch.log(torch.where(valid, q, 1.0))
    loss = w * tau * tau * (q * (logq - logp)).sum(1)
    if not c["grad"]:
        return {"loss": loss, "dlogits": None}
    d = e / S
    d.scatter_add_(1, at, -q)
    return {"loss": loss, "dlogits": (d * (w * tau)[:, None]).to(s["logits"].dtype)}


def _top_plain(logits, k):
    """Indices of the k largest, equal ones in the order of their index."""
    bits = logits.float().add(0.0).view(torch.int32).long()        # + 0: one zero
    key = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits) << 32  # increasing with the value
    return torch.topk(key - torch.arange(logits.shape[1], device=logits.device), k, dim=1).indices


# ---- work and 64-bit values -----------------------------------------------------------------------
def work(case):
    c = case
    size = lambda name: _TYPES[name].itemsize  # noqa: E731
    op = c["op"]
    if op == "norm":
        n, b = c["T"] * c["H"], size(c["type"])
        return {"bytes": n * (3 * b + 1) + n // 128 + c["H"] * b + 4 * c["T"] * c["train"], "flops": 8 * n}
    if op == "norm_bwd":
        n, b = c["T"] * c["H"], size(c["type"])
        return {"bytes": n * 4 * b + c["H"] * (b + 4) + 4 * c["T"], "flops": 11 * n}
    if op == "cut":
        n, copies = c["M"] * c["K"], 2 if c["both"] else 1
        return {"bytes": n * (size(c["type"]) + copies) + copies * n // (128 * c["block_rows"]), "flops": 3 * copies * n}
    if op == "product":
        M, N, K = c["M"], c["N"], c["K"]
        return {"bytes": (M + N) * K + M * K // 128 + N * K // (128 * c["b_rows"]) + M * N * size(c["out"]),
                "flops": 2 * M * N * K}
    n, b = c["T"] * c["V"], size(c["type"])
    if op == "logprobs":
        return {"bytes": n * b + c["T"] * (16 + 8 * c["top"]), "flops": 6 * n}
    if op == "logprobs_bwd":
        # the logits are read twice: the upstream gradients may depend on the forward pass's results
        return {"bytes": 3 * n * b + c["T"] * 36, "flops": 14 * n}
    return {"bytes": n * b * (2 if c["grad"] else 1) + c["T"] * (8 + 8 * c["K"]), "flops": (8 if c["grad"] else 4) * n}


def _cut_exact(x, name, block_rows):
    """Elements over their block's scale, before they are rounded to 8 bits."""
    rows, cols = x.shape
    big = torch.zeros(((rows + block_rows - 1) // block_rows, (cols + 127) // 128), dtype=x.dtype, device=x.device)
    for j in range(big.shape[1]):
        part = x[:, 128 * j:128 * (j + 1)].abs().amax(1)
        big[:, j].scatter_reduce_(0, torch.arange(rows, device=x.device) // block_rows, part, "amax", include_self=True)
    scale = torch.where(big > 0, torch.exp2(torch.ceil(torch.log2(big / _TOP[name]))), 1.0)
    row, col = torch.arange(rows, device=x.device) // block_rows, torch.arange(cols, device=x.device) // 128
    return x / scale[row][:, col]


def exact(case, seed):
    s, c = prepare(case, seed), case
    op = c["op"]
    if op == "norm":
        h = s["x"].double() + s["residual"].double()
        rstd = (h.pow(2).sum(1) / c["H"] + _EPS).pow(-0.5)
        y = torch.einsum("th,t,h->th", h, rstd, s["weight"].double())
        return {"residual": h, "q": _cut_exact(y, c["q"], 1), "scales": None, "rstd": rstd if c["train"] else None}
    if op == "norm_bwd":
        h, dy, r = s["h"].double(), s["dy"].double(), s["rstd"].double()
        g = dy * s["weight"].double()
        dx = g * r[:, None] - h * (r.pow(3) * torch.einsum("th,th->t", g, h) / c["H"])[:, None] + s["dresidual"].double()
        return {"dx": dx, "dweight": torch.einsum("th,th,t->h", dy, h, r)}
    if op == "cut":
        x = s["src"].double()
        return {"q": _cut_exact(x, c["q"], c["block_rows"]), "scales": None, "scalesT": None,
                "qT": _cut_exact(x.t(), c["q"], c["block_rows"]) if c["both"] else None}
    if op == "product":
        col = torch.arange(c["K"], device="cuda") // 128
        row = torch.arange(c["N"], device="cuda") // c["b_rows"]
        A = s["A"].double() * s["a_scales"].double()[:, col]
        B = s["B"].double() * s["b_scales"].double()[row][:, col]
        return torch.einsum("mk,nk->mn", A, B)
    z = s["logits"].double() / c["temperature"]
    lse = torch.logsumexp(z, 1)
    logp = z - lse[:, None]
    if op in ("logprobs", "logprobs_bwd"):
        p = logp.exp()
        H = -(p * logp).sum(1)
        at = s["tokens"].long()
        rows = torch.arange(c["T"], device="cuda")
        out = {"logprobs": logp[rows, at], "lse": lse, "entropy": H}
        if op == "logprobs":
            top = torch.sort(logp, dim=1, descending=True).values[:, :c["top"]] if c["top"] else None
            return {**out, "top_ids": None, "top_logprobs": top}
        gl, gh = s["dlogprobs"].double(), s["dentropy"].double()
        d = -p * (gl[:, None] + gh[:, None] * (logp + H[:, None]))
        d[rows, at] += gl
        return {**out, "dlogits": d / c["temperature"]}
    tau, w = c["temperature"], s["weights"].double()
    valid = s["teacher_ids"] >= 0
    at = s["teacher_ids"].clamp(min=0).long()
    logq = torch.log_softmax(s["teacher_logits"].double().div(tau).masked_fill(~valid, -math.inf), 1)
    q = logq.exp()
    loss = (q * (logq.masked_fill(~valid, 0.0) - logp.gather(1, at))).sum(1) * w * tau ** 2
    if not c["grad"]:
        return {"loss": loss, "dlogits": None}
    d = logp.exp_()
    d.scatter_add_(1, at, -q)
    return {"loss": loss, "dlogits": d * (w * tau)[:, None]}
