"""Cases, plain forms and calls of the adapter, head-norm and gradient-clipping operators.

The operators are those between and after the 8-bit projections of a language model that is fine-tuned with
low-rank adapters or serves many of them at once: the adapters beside a shared projection, the norms of queries
and keys for each head with the rotation by position in the same pass, and the norm over many gradients with the
clipping by it.

Adapters: the rows (tokens) of a batch are cut into segments (requests); segment s covers the rows offsets[s] up
to offsets[s + 1] and has the adapter index[s], -1 for none.  With x [T, K], A [n, r, K], B [n, N, r], base [T, N]

    h[t] = A_i x[t],    out[t] = base[t] + scale_i B_i h[t],

h being zero in rows without an adapter.  Rotation: pair j of a head's first R columns (columns j and j + R / 2, or
2 j and 2 j + 1 where neighbours are paired) turns by the angle whose cosine and sine stand in the columns j and
R / 2 + j of a table's row; the row is the token's position, along the pair's axis where positions have several.
Clipping: every gradient times min(1, max_norm / norm), the norm taken over all of them together.

`run` with `own` false computes the operators from elementary torch operations in 32 bits, rounded once; with `own`
true it makes the calls of the framework.  `exact` gives the same outputs from the definitions in 64 bits.
"""

import math
import random

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_EPS = 1e-6


# ---- cases ----------------------------------------------------------------------------------------
def listed():
    return [
        # queries and keys of eight sequences that produce one token each: latency
        dict(name="heads decode", op="heads", T=8, Hq=32, Hk=8, D=128, R=128, P=32768, axes=1, neighbours=False, norm=True, type="bf16"),
        # a long batch of prompts, many query heads
        dict(name="heads prompts", op="heads", T=16384, Hq=64, Hk=8, D=128, R=128, P=131072, axes=1, neighbours=False, norm=True, type="bf16"),
        # patches of a video (time, height, width), rotation alone, narrow heads, odd number of tokens
        dict(name="heads video", op="heads", T=5003, Hq=16, Hk=16, D=80, R=80, P=2048, axes=3, neighbours=True, norm=False, type="f16"),
        # the gradient in a training step of a middle-sized layer
        dict(name="heads backward", op="heads_bwd", T=4096, Hq=32, Hk=8, D=128, R=128, P=8192, axes=1, neighbours=False, norm=True, type="bf16"),
        # 64 requests, each with an adapter of its own, produce one token each: reads the adapters, little else
        dict(name="adapters decode", op="adapters", T=64, S=64, n=64, r=16, K=4096, N=4096, type="bf16", out="bf16", without=False),
        # a batch of ragged prompts beside a fused projection, a few requests without an adapter
        dict(name="adapters prompts", op="adapters", T=4001, S=12, n=9, r=64, K=4096, N=6144, type="bf16", out="bf16", without=True),
        # one adapter being evaluated over a large batch
        dict(name="adapters large", op="adapters", T=16384, S=24, n=4, r=32, K=8192, N=8192, type="bf16", out="bf16", without=False),
        # fine-tuning of one adapter: gradients of the input and, in FP32, of both factors
        dict(name="adapters training", op="adapters_bwd", T=8192, S=1, n=1, r=16, K=4096, N=4096, type="bf16", out="bf16", grad="f32"),
        # three adapters trained side by side, wide output, gradients in their own type, odd number of tokens
        dict(name="adapters training of three", op="adapters_bwd", T=2050, S=7, n=3, r=64, K=4096, N=11008, type="bf16", out="bf16", grad="bf16"),
        # the gradients of a small model's adapters: latency of many small tensors
        dict(name="clip adapters", op="clip", count=56, total=56 * 16 * 2048, type="f32", loud=True, even=True),
        # FP32 and BF16 gradients of odd sizes
        dict(name="clip mixed", op="clip", count=37, total=30000007, type="mixed", loud=True),
        # all gradients of a model of 400 million weights
        dict(name="clip model", op="clip", count=290, total=400000000, type="bf16", loud=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    op = rng.choice(["heads", "heads", "heads_bwd", "adapters", "adapters", "adapters", "adapters_bwd", "adapters_bwd", "clip", "clip"])
    t = rng.choice(["bf16", "bf16", "f16"])
    if op in ("heads", "heads_bwd"):
        t = rng.choice([t, t, t, "f32"])
        D = rng.choice([64, 80, 128, 128, 128, 256])
        Hk = rng.choice([1, 2, 4, 8])
        Hq = Hk * rng.choice([1, 4, 5, 8])
        T = _log(rng, 1, 16384 * 72 * 128 // (max(72, Hq + Hk) * max(D, 128)))
        c = dict(op=op, T=T, Hq=Hq, Hk=Hk, D=D, R=rng.choice([D, D, D // 2]), P=rng.choice([4096, 32768, 131072]),
                 axes=rng.choice([1, 1, 1, 3]), neighbours=rng.random() < 0.3, norm=rng.random() < 0.8, type=t)
        return c
    if op == "clip":
        count = _log(rng, 1, 400)
        return dict(op=op, count=count, total=max(count, _log(rng, 1000, 200000000)), type=rng.choice(["f32", "bf16", "f16", "mixed"]),
                    loud=rng.random() < 0.7)
    r = rng.choice([4, 8, 16, 16, 32, 64, 64, 7, 128])
    K, N = _log(rng, 256, 12000), _log(rng, 256, 12000)
    if rng.random() < 0.8:                                         # layers are seldom odd
        K, N = K // 64 * 64, N // 64 * 64
    out = rng.choice([t, t, "f32"])
    if op == "adapters":
        T = _log(rng, 1, min(16384, 16384 * 24576 // (K + 2 * N)))
        S = T if T <= 256 and rng.random() < 0.5 else _log(rng, 1, min(T, 64))
        return dict(op=op, T=T, S=S, n=_log(rng, 1, min(S, 64)), r=r, K=K, N=N, type=t, out=out, without=rng.random() < 0.3)
    T = _log(rng, 16, 8192)
    S = _log(rng, 1, min(T, 32))
    return dict(op=op, T=T, S=S, n=_log(rng, 1, min(S, 8)), r=r, K=K, N=N, type=t, out=t, grad=rng.choice(["f32", t]))


# ---- inputs ---------------------------------------------------------------------------------------
def _segments(case, seed):
    """[(first row, end, adapter)]: requests of uneven length in one batch; every adapter is used where segments suffice."""
    rng = random.Random(seed * 7919 + case["T"])
    T, S, n = case["T"], case["S"], case["n"]
    cuts = list(range(T + 1)) if S == T else [0] + sorted(rng.randint(0, T) for _ in range(S - 1)) + [T]
    ids = [i % n for i in range(S)]
    rng.shuffle(ids)
    if case.get("without"):
        ids = [-1 if i % 8 == 5 else a for i, a in enumerate(ids)]
    return list(zip(cuts[:-1], cuts[1:], ids))


def _sizes(case):
    """Element counts of the gradients: a few large and many small ones, or all alike."""
    if case.get("even"):
        return [case["total"] // case["count"]] * case["count"]
    rng = random.Random(case["count"] * 1000003 + case["total"])
    w = [math.exp(rng.gauss(0.0, 1.5)) for _ in range(case["count"])]
    sizes = [max(1, int(case["total"] * v / sum(w))) for v in w]
    sizes[sizes.index(max(sizes))] += max(0, case["total"] - sum(sizes))
    return sizes


def _grad_types(case):
    names = ["f32", "bf16", "bf16"] if case["type"] == "mixed" else [case["type"]]
    return [_TYPES[names[i % len(names)]] for i in range(case["count"])]


def _table(P, R):
    """Cosines and sines of every position and pair, angles in 64 bits."""
    f = torch.exp(torch.arange(R // 2, device="cuda", dtype=torch.float64) * (-2.0 / R * math.log(10000.0)))
    a = torch.arange(P, device="cuda", dtype=torch.float64)[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float()


def _prepare_heads(c, rand, gen, s):
    T, Hq, Hk, D, R, P, dt = c["T"], c["Hq"], c["Hk"], c["D"], c["R"], c["P"], _TYPES[c["type"]]
    # queries and keys as the fused projection leaves them, the values behind
    fused = (rand(T, (Hq + 2 * Hk) * D) * torch.exp(rand(1, (Hq + 2 * Hk) * D) * 0.5)).to(dt)
    s["q"], s["k"] = fused[:, :Hq * D], fused[:, Hq * D:(Hq + Hk) * D]
    s["q_weight"], s["k_weight"] = [(1 + 0.1 * rand(D)).to(dt) for _ in range(2)] if c["norm"] else (None, None)
    s["table"] = _table(P, R)
    if c["axes"] == 1:                                             # sequences of consecutive positions, or one token of each
        if T <= 64:
            s["positions"] = torch.randint(0, P, (T,), device="cuda", generator=gen, dtype=torch.int32)
        else:
            start = int(torch.randint(0, max(1, P - T), (1,), device="cuda", generator=gen))
            s["positions"] = ((torch.arange(T, device="cuda") + start) % P).to(torch.int32)
        s["axes"] = None
    else:                                                          # time, rows and columns of patches, frequencies dealt out in turn
        t = torch.arange(T, device="cuda")
        s["positions"] = (torch.stack([t // 1564, t // 46 % 34, t % 46], 1) % P).to(torch.int32)
        s["axes"] = (torch.arange(R // 2, device="cuda") % 3).to(torch.uint8)
    if c["op"] == "heads":
        s["q_out"], s["k_out"] = (torch.empty((T, h * D), device="cuda", dtype=dt) for h in (Hq, Hk))
        return
    s["dq"], s["dk"] = ((1e-2 * rand(T, h * D)).to(dt) for h in (Hq, Hk))
    s["dx"] = torch.empty((T, (Hq + Hk) * D), device="cuda", dtype=dt)
    if c["norm"]:
        s["dq_weight"], s["dk_weight"] = torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
        s["workspace"] = torch.empty(1024 * D, device="cuda")      # FP32 rows of partial sums, 512 for each weight


def _prepare_adapters(c, rand, seed, s):
    T, n, r, K, N, dt, out = c["T"], c["n"], c["r"], c["K"], c["N"], _TYPES[c["type"]], _TYPES[c["out"]]
    s["segments"] = _segments(c, seed)
    s["offsets"] = torch.tensor([a for a, _, _ in s["segments"]] + [T], device="cuda", dtype=torch.int32)
    s["index"] = torch.tensor([i for _, _, i in s["segments"]], device="cuda", dtype=torch.int32)
    s["x"] = rand(T, K).to(dt)
    s["A"], s["B"] = (rand(n, r, K) / math.sqrt(K)).to(dt), (rand(n, N, r) / math.sqrt(r)).to(dt)
    s["scale"] = torch.full((n,), 2.0, device="cuda") + 0.25 * torch.arange(n, device="cuda") / n
    s["h"] = torch.empty((T, r), device="cuda")
    if c["op"] == "adapters":
        s["base"] = rand(T, N).to(out)                             # what the shared projection gave
        s["out"] = torch.empty((T, N), device="cuda", dtype=out)
        return
    s["h"] = torch.cat([s["x"][a:b].float() @ s["A"][i].float().t() for a, b, i in s["segments"]])
    s["dout"] = (1e-2 * rand(T, N)).to(out)
    s["dbase"] = (1e-2 * rand(T, K)).to(dt)                        # the shared projection's share of the input's gradient
    s["dx"] = torch.empty((T, K), device="cuda", dtype=dt)
    s["dA"], s["dB"] = (torch.empty(shape, device="cuda", dtype=_TYPES[c["grad"]]) for shape in ((n, r, K), (n, N, r)))
    s["workspace"] = torch.empty(512 << 20, device="cuda", dtype=torch.uint8)


def _flat(c, sizes, dtype=None):
    """The buffers that an optimizer keeps, one for each type, and where in them each gradient goes: on 128-byte boundaries."""
    at, end = [], {}
    for k, t in zip(sizes, _grad_types(c)):
        at.append((t, end.get(t, 0), k))
        end[t] = end.get(t, 0) + (k + 127) // 128 * 128
    flat = {t: torch.zeros(n, device="cuda", dtype=dtype or t) for t, n in end.items()}
    return flat, [flat[t][a:a + k] for t, a, k in at]


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    rand = lambda *shape: torch.randn(shape, device="cuda", generator=gen)  # noqa: E731
    s = {"case": c}
    if c["op"] in ("heads", "heads_bwd"):
        _prepare_heads(c, rand, gen, s)
    elif c["op"] in ("adapters", "adapters_bwd"):
        _prepare_adapters(c, rand, int(seed), s)
    else:
        # layers' gradients differ in size by what sits above them
        sizes = _sizes(c)
        level = (4.0 if c["loud"] else 0.3) / math.sqrt(sum(sizes))
        s["grads"] = [(rand(k) * level * (0.5 + (i % 7) / 4)).to(t) for i, (k, t) in enumerate(zip(sizes, _grad_types(c)))]
        s["flat"], s["clipped"] = _flat(c, sizes)
        s["norm"] = torch.empty(1, device="cuda")
        s["workspace"] = torch.empty(1 << 16, device="cuda", dtype=torch.uint8)
    return s


# ---- one pass -------------------------------------------------------------------------------------
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    import paper_1811_10751_b200 as g
    c = s["case"]
    op = c["op"]
    if op == "heads":
        g.gpd_head_norm_rope(s["q"], s["k"], s["table"], s["positions"], s["q_out"], s["k_out"], c["D"], q_weight=s["q_weight"],
                             k_weight=s["k_weight"], eps=_EPS, axes=s["axes"], neighbours=c["neighbours"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if op == "heads_bwd":
        Hq, D = c["Hq"], c["D"]
        g.gpd_head_norm_rope_backward(s["dq"], s["dk"], s["q"], s["k"], s["table"], s["positions"], s["dx"][:, :Hq * D],
                                      s["dx"][:, Hq * D:], D, q_weight=s["q_weight"], k_weight=s["k_weight"],
                                      dq_weight=s.get("dq_weight"), dk_weight=s.get("dk_weight"), workspace=s.get("workspace"),
                                      eps=_EPS, axes=s["axes"], neighbours=c["neighbours"])
        return {k: s.get(k) for k in ("dx", "dq_weight", "dk_weight")}
    if op == "adapters":
        g.gpd_adapter(s["x"], s["A"], s["B"], s["offsets"], s["index"], s["out"], s["h"], base=s["base"], scale=s["scale"])
        return {"out": s["out"], "h": s["h"]}
    if op == "adapters_bwd":
        g.gpd_adapter_backward(s["dout"], s["x"], s["A"], s["B"], s["h"], s["offsets"], s["index"], s["dx"], s["dA"], s["dB"],
                               s["workspace"], dbase=s["dbase"], scale=s["scale"])
        return {k: s[k] for k in ("dx", "dA", "dB")}
    g.gpd_grad_norm(s["grads"], s["norm"], s["workspace"])
    g.gpd_clip_grads(s["grads"], s["norm"], 1.0, out=s["clipped"])
    return {"norm": s["norm"], "grads": list(s["flat"].values())}


def _angles(s):
    """Cosines and sines [T, 1, R / 2] of every token's pairs."""
    half = s["table"].shape[1] // 2
    if s["axes"] is None:
        row = s["table"][s["positions"].long()]
        return row[:, None, :half], row[:, None, half:]
    at, j = s["positions"].long()[:, s["axes"].long()], torch.arange(half, device="cuda")
    return s["table"][at, j][:, None], s["table"][at, j + half][:, None]


def _turn(x, cos, sin, neighbours):
    """x [T, H, D], its pairs turned."""
    half = cos.shape[-1]
    a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if neighbours else (x[..., :half], x[..., half:2 * half])
    u, v = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([u, v], -1).flatten(-2) if neighbours else torch.cat([u, v], -1)
    return torch.cat([turned, x[..., 2 * half:]], -1)


def _heads_plain(x, w, cos, sin, c):
    x = x.float().reshape(c["T"], -1, c["D"])
    if w is not None:
        x = x * torch.rsqrt(x.square().mean(2, keepdim=True) + _EPS) * w.float()
    return _turn(x, cos, sin, c["neighbours"]).flatten(1)


def _heads_bwd_plain(dy, x, w, cos, sin, c):
    g = _turn(dy.float().reshape(c["T"], -1, c["D"]), cos, -sin, c["neighbours"])
    if w is None:
        return g.flatten(1), None
    x = x.float().reshape(c["T"], -1, c["D"])
    r = torch.rsqrt(x.square().mean(2, keepdim=True) + _EPS)
    n, gw = x * r, g * w.float()
    return (r * (gw - n * (gw * n).mean(2, keepdim=True))).flatten(1), (g * n).sum((0, 1))


def _run_plain(s):
    c = s["case"]
    op = c["op"]
    if op in ("heads", "heads_bwd"):
        cos, sin = _angles(s)
        if op == "heads":
            return {"q": _heads_plain(s["q"], s["q_weight"], cos, sin, c).to(s["q"].dtype),
                    "k": _heads_plain(s["k"], s["k_weight"], cos, sin, c).to(s["q"].dtype)}
        dq, dwq = _heads_bwd_plain(s["dq"], s["q"], s["q_weight"], cos, sin, c)
        dk, dwk = _heads_bwd_plain(s["dk"], s["k"], s["k_weight"], cos, sin, c)
        return {"dx": torch.cat([dq.to(s["q"].dtype), dk.to(s["q"].dtype)], 1), "dq_weight": dwq, "dk_weight": dwk}
    if op == "adapters":
        parts = [_adapter_plain(s["x"][a:b], s["A"], s["B"], s["scale"], i) for a, b, i in s["segments"]]
        out = s["base"].float() + torch.cat([d for d, _ in parts])
        return {"out": out.to(s["out"].dtype), "h": torch.cat([h for _, h in parts])}
    if op == "adapters_bwd":
        parts = [(i, s["x"][a:b].float(), s["h"][a:b], s["scale"][i] * s["dout"][a:b].float()) for a, b, i in s["segments"]]
        g = [(i, x, h, d, d @ s["B"][i].float()) for i, x, h, d in parts]
        dx = s["dbase"].float() + torch.cat([u @ s["A"][i].float() for i, _, _, _, u in g])
        dA, dB = torch.zeros(s["dA"].shape, device="cuda"), torch.zeros(s["dB"].shape, device="cuda")
        at = s["index"].long()
        dA.index_add_(0, at, torch.stack([u.t() @ x for _, x, _, _, u in g]))
        dB.index_add_(0, at, torch.stack([d.t() @ h for _, _, h, d, _ in g]))
        return {"dx": dx.to(s["dx"].dtype), "dA": dA.to(s["dA"].dtype), "dB": dB.to(s["dB"].dtype)}
    norm = torch.stack([x.float().square().sum(dtype=torch.float64) for x in s["grads"]]).sum().sqrt().float()
    by = torch.clamp(1.0 / norm, max=1.0)
    torch._foreach_copy_(s["clipped"], [x.float() * by for x in s["grads"]])
    return {"norm": norm[None], "grads": list(s["flat"].values())}


def _adapter_plain(x, A, B, scale, i):
    if i < 0:
        return torch.zeros((x.shape[0], B.shape[1]), device="cuda"), torch.zeros((x.shape[0], A.shape[1]), device="cuda")
    h = x.float() @ A[i].float().t()
    return scale[i] * (h @ B[i].float().t()), h


# ---- work and 64-bit values -----------------------------------------------------------------------
def work(case):
    c = case
    op = c["op"]
    if op in ("heads", "heads_bwd"):
        b, T, D = _TYPES[c["type"]].itemsize, c["T"], c["D"]
        n = T * (c["Hq"] + c["Hk"]) * D
        rest = min(T, c["P"]) * c["R"] * 4 + T * c["axes"] * 4
        if op == "heads":
            return {"bytes": 2 * n * b + rest + 2 * D * b * c["norm"], "flops": n * (3 + 4 * c["norm"])}
        moved = 3 if c["norm"] else 2                              # the rotation's gradient does not need its input
        return {"bytes": moved * n * b + rest + 2 * D * (b + 4) * c["norm"], "flops": n * (3 + 11 * c["norm"])}
    if op == "clip":
        sizes, types = _sizes(c), _grad_types(c)
        return {"bytes": 2 * sum(k * t.itemsize for k, t in zip(sizes, types)) + 4, "flops": 3 * sum(sizes)}
    T, n, r, K, N = c["T"], c["n"], c["r"], c["K"], c["N"]
    b, o, tables = _TYPES[c["type"]].itemsize, _TYPES[c["out"]].itemsize, 8 * c["S"] + 4
    if op == "adapters":
        return {"bytes": T * (K * b + 2 * N * o + 4 * r) + n * r * (K + N) * b + tables + 4 * n, "flops": 2 * T * r * (K + N)}
    g = _TYPES[c["grad"]].itemsize
    return {"bytes": T * (3 * K * b + N * o + 4 * r) + n * r * (K + N) * (b + g) + tables + 4 * n, "flops": 4 * T * r * (K + N)}


def _heads_exact(x, w, s):
    """By complex numbers."""
    c, half = s["case"], s["table"].shape[1] // 2
    x = x.reshape(c["T"], -1, c["D"])
    if w is not None:
        x = x / torch.sqrt((x * x).sum(2, keepdim=True) / c["D"] + _EPS) * w
    pos = s["positions"].long().view(c["T"], -1)
    axis = s["axes"].long() if s["axes"] is not None else torch.zeros(half, dtype=torch.long, device="cuda")
    cols = torch.arange(half, device="cuda")
    t = s["table"].double()
    unit = torch.complex(t[pos[:, axis], cols], t[pos[:, axis], cols + half])[:, None]
    first = 2 * cols if c["neighbours"] else cols
    second = first + (1 if c["neighbours"] else half)
    z = torch.complex(x[..., first], x[..., second]) * unit
    y = x.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y.reshape(c["T"], -1)


def exact(case, seed):
    s, c = prepare(case, seed), case
    op = c["op"]
    if op == "heads":
        return {k: _heads_exact(s[k].double(), s[k + "_weight"].double() if c["norm"] else None, s) for k in ("q", "k")}
    if op == "heads_bwd":
        dx, dw = [], []
        for k in ("q", "k"):
            x = s[k].double().requires_grad_()
            w = s[k + "_weight"].double().requires_grad_() if c["norm"] else None
            _heads_exact(x, w, s).backward(s["d" + k].double())
            dx.append(x.grad)
            dw.append(w.grad if c["norm"] else None)
        return {"dx": torch.cat(dx, 1), "dq_weight": dw[0], "dk_weight": dw[1]}
    if op == "clip":
        norm = torch.sqrt(sum(torch.dot(v, v) for v in (x.double() for x in s["grads"])))
        by = 1.0 / norm if norm > 1.0 else torch.ones_like(norm)
        flat, parts = _flat(c, _sizes(c), torch.float64)
        for part, x in zip(parts, s["grads"]):
            part.copy_(x.double() * by)
        return {"norm": norm[None], "grads": list(flat.values())}
    if op == "adapters":
        out, h = s["base"].double(), torch.zeros((c["T"], c["r"]), device="cuda", dtype=torch.float64)
        for a, b, i in s["segments"]:
            if i >= 0:
                h[a:b] = torch.einsum("tk,rk->tr", s["x"][a:b].double(), s["A"][i].double())
                out[a:b] += torch.einsum("tr,nr->tn", h[a:b], s["scale"][i].double() * s["B"][i].double())
        return {"out": out, "h": h}
    dx = s["dbase"].double()
    dA, dB = (torch.zeros(s[k].shape, device="cuda", dtype=torch.float64) for k in ("dA", "dB"))
    for a, b, i in s["segments"]:
        d = s["dout"][a:b].double() * s["scale"][i].double()
        u = torch.einsum("tn,nr->tr", d, s["B"][i].double())
        dx[a:b] += torch.einsum("tr,rk->tk", u, s["A"][i].double())
        dA[i] += torch.einsum("tr,tk->rk", u, s["x"][a:b].double())
        dB[i] += torch.einsum("tn,tr->nr", d, s["h"][a:b].double())
    return {"dx": dx, "dA": dA, "dB": dB}
