"""Queries and keys of one layer with adapters: serving several fine-tuned forms of a model at once, and a training step.

serving:   8-bit projection that all requests share + each request's low-rank adapter -> norms of queries and keys per head and
           their rotation by position
training:  the same, then back: gradients through rotation and norms -> gradients of both factors of the adapters and of the
           hidden states (on top of the shared projection's) -> norm over all gradients, clipping -> a step

Run:  python examples/adapter_step.py [--tokens T] [--hidden H] [--rank R]
Prints, for each result, how far it is from the same step in FP32 (with the projection's weights as 8 bits hold them).
"""

from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1811_10751_b200 as g  # noqa: E402

E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2


class AdaptedHeads:
    """Queries and keys [T, (q_heads + k_heads) head_dim] from hidden states [T, H]: a frozen 8-bit projection, adapters A [n, r, H]
    and B [n, N, r] beside it, norms per head with their weights, rotation by position.  Buffers are kept from step to step."""

    def __init__(self, weight, A, B, scale, q_weight, k_weight, q_heads: int, k_heads: int, head_dim: int, tokens: int, positions: int):
        N, H = weight.shape
        n, r, _ = A.shape
        dev = weight.device
        self.A, self.B, self.scale, self.q_weight, self.k_weight = A, B, scale, q_weight, k_weight
        self.D, self.split = head_dim, q_heads * head_dim
        assert N == (q_heads + k_heads) * head_dim
        self.w, self.w_scales = g.new_fp8(N, H, E4M3, 128, device=dev)
        self.wT, self.wT_scales = g.new_fp8(H, N, E4M3, 128, device=dev)
        g.gpd_quantize_blocks(weight, q=self.w, scales=self.w_scales, qT=self.wT, scalesT=self.wT_scales, block_rows=128)
        self.table = g.new_rope_table(positions, head_dim, device=dev)
        make = lambda *s, dtype=torch.bfloat16: torch.empty(s, dtype=dtype, device=dev)  # noqa: E731
        self.x8, self.x8_scales = g.new_fp8(tokens, H, device=dev)
        self.raw, self.h = make(tokens, N), make(tokens, r, dtype=torch.float32)
        self.out, self.d = make(tokens, N), make(tokens, N)
        self.d8, self.d8_scales = g.new_fp8(tokens, N, E5M2, device=dev)
        self.dx = make(tokens, H)
        self.dA, self.dB = make(n, r, H, dtype=torch.float32), make(n, N, r, dtype=torch.float32)
        self.dq_weight, self.dk_weight = make(head_dim, dtype=torch.float32), make(head_dim, dtype=torch.float32)
        self.heads_ws = make(2 * g.GPD_HEAD_NORM_MAX_PARTS * head_dim, dtype=torch.float32)
        self.adapter_ws = make(g.gpd_adapter_backward_workspace(tokens, H, N, n, r), dtype=torch.uint8)
        self.norm, self.norm_ws = make(1, dtype=torch.float32), make(g.GPD_GRAD_NORM_WORKSPACE, dtype=torch.uint8)

    def _parts(self, m):
        return m[:, :self.split], m[:, self.split:]

    def forward(self, x, positions, offsets, index):
        """x: [T, H] BF16; requests' rows offsets[s] .. offsets[s + 1] have the adapter index[s], -1 for none."""
        g.gpd_quantize_blocks(x, q=self.x8, scales=self.x8_scales)
        g.gpd_gemm_fp8(self.x8, self.x8_scales, self.w, self.w_scales, self.raw)
        g.gpd_adapter(x, self.A, self.B, offsets, index, self.raw, self.h, base=self.raw, scale=self.scale)
        (q, k), (qo, ko) = self._parts(self.raw), self._parts(self.out)
        g.gpd_head_norm_rope(q, k, self.table, positions, qo, ko, self.D, q_weight=self.q_weight, k_weight=self.k_weight)
        return qo, ko

    def backward(self, dq, dk, x, positions, offsets, index):
        """Gradient of x; those of the adapters and of the heads' weights stay in dA, dB, dq_weight and dk_weight."""
        (q, k), (dqi, dki) = self._parts(self.raw), self._parts(self.d)
        g.gpd_head_norm_rope_backward(dq, dk, q, k, self.table, positions, dqi, dki, self.D, q_weight=self.q_weight, k_weight=self.k_weight,
                                      dq_weight=self.dq_weight, dk_weight=self.dk_weight, workspace=self.heads_ws)
        g.gpd_quantize_blocks(self.d, q=self.d8, scales=self.d8_scales)
        g.gpd_gemm_fp8(self.d8, self.d8_scales, self.wT, self.wT_scales, self.dx)
        g.gpd_adapter_backward(self.d, x, self.A, self.B, self.h, offsets, index, self.dx, self.dA, self.dB, self.adapter_ws,
                               dbase=self.dx, scale=self.scale)
        return self.dx

    def clip(self, max_norm: float):
        """Gradients to a common norm of at most max_norm; returns the norm before."""
        grads = [self.dA, self.dB, self.dq_weight, self.dk_weight]
        g.gpd_grad_norm(grads, self.norm, self.norm_ws)
        g.gpd_clip_grads(grads, self.norm, max_norm)
        return self.norm

    def step(self, rate: float):
        self.A.add_(self.dA.to(self.A.dtype), alpha=-rate)
        self.B.add_(self.dB.to(self.B.dtype), alpha=-rate)
        self.q_weight.add_(self.dq_weight.to(self.q_weight.dtype), alpha=-rate)
        self.k_weight.add_(self.dk_weight.to(self.k_weight.dtype), alpha=-rate)


def fp32_step(weight, A, B, scale, q_weight, k_weight, head_dim, split, x, positions, segments, dq, dk, eps=1e-6):
    """The same by automatic differentiation in FP32 (angles in FP64)."""
    x, A, B, qw, kw = (t.detach().float().requires_grad_() for t in (x, A, B, q_weight, k_weight))
    out = x @ weight.float().t()
    parts = [out[a:b] + (scale[i] * (x[a:b] @ A[i].t()) @ B[i].t() if i >= 0 else 0.0) for a, b, i in segments]
    out = torch.cat(parts)
    j = torch.arange(head_dim // 2, device=x.device, dtype=torch.float64)
    angle = positions.double()[:, None] * 10000.0 ** (-2 * j / head_dim)
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def heads(z, w):
        z = z.view(z.shape[0], -1, head_dim)
        z = z * torch.rsqrt(z.square().mean(2, keepdim=True) + eps) * w
        a, b = z.chunk(2, 2)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], 2).flatten(1)
    q, k = heads(out[:, :split], qw), heads(out[:, split:], kw)
    ((q * dq.float()).sum() + (k * dk.float()).sum()).backward()
    return q.detach(), k.detach(), x.grad, A.grad, B.grad, qw.grad, kw.grad


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--tokens", type=int, default=1000)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--rank", type=int, default=16)
    a = ap.parse_args(argv)
    q_heads, k_heads, D, n, requests = 8, 2, 128, 3, 6
    N, T, H, r = (q_heads + k_heads) * D, a.tokens, a.hidden, a.rank
    gen = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    weight = (rand(N, H) / H ** 0.5).bfloat16()
    A, B = (rand(n, r, H) / H ** 0.5).bfloat16(), (rand(n, N, r) / r ** 0.5).bfloat16()
    scale = torch.tensor([0.5, 1.0, 2.0], device="cuda")
    qw, kw = (1 + 0.1 * rand(D)).bfloat16(), (1 + 0.1 * rand(D)).bfloat16()
    x, positions = rand(T, H).bfloat16(), torch.randint(0, 4096, (T,), device="cuda", generator=gen)
    dq, dk = rand(T, q_heads * D).bfloat16(), rand(T, k_heads * D).bfloat16()
    cuts = sorted(torch.randint(0, T + 1, (requests - 1,), generator=torch.Generator().manual_seed(2)).tolist())
    cuts, index = [0] + cuts + [T], [0, 2, -1, 1, 0, 2]
    offsets, index_dev = torch.tensor(cuts, device="cuda"), torch.tensor(index, device="cuda")
    segments = list(zip(cuts[:-1], cuts[1:], index))

    layer = AdaptedHeads(weight, A, B, scale, qw, kw, q_heads, k_heads, D, T, 4096)
    q, k = layer.forward(x, positions, offsets, index_dev)
    dx = layer.backward(dq, dk, x, positions, offsets, index_dev)
    grads = [t.clone() for t in (layer.dA, layer.dB, layer.dq_weight, layer.dk_weight)]
    norm = layer.clip(1.0)

    seen = layer.w.float() * torch.exp2(layer.w_scales.view(torch.uint8).float() - 127).repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :H]
    ref = fp32_step(seen, A, B, scale, qw, kw, D, q_heads * D, x, positions, segments, dq, dk)
    off = lambda got, want: float((got.float() - want).norm() / want.norm())  # noqa: E731
    far = {"queries": off(q, ref[0]), "keys": off(k, ref[1]), "d hidden": off(dx, ref[2]), "d A": off(grads[0], ref[3]),
           "d B": off(grads[1], ref[4]), "d query weight": off(grads[2], ref[5]), "d key weight": off(grads[3], ref[6])}
    want = torch.sqrt(sum(t.double().square().sum() for t in grads))
    far["norm"] = abs(float(norm) / float(want) - 1)
    far["clipped"] = abs(float(torch.sqrt(sum(t.double().square().sum() for t in (layer.dA, layer.dB, layer.dq_weight, layer.dk_weight)))) - 1)
    layer.step(1e-2)
    assert g.gpd_device_status() == 0

    # serving: the same layer, one token of each of 40 requests
    S = 40
    serve = AdaptedHeads(weight, layer.A, layer.B, scale, layer.q_weight, layer.k_weight, q_heads, k_heads, D, S, 4096)
    one = [i % (n + 1) - 1 for i in range(S)]
    q1, k1 = serve.forward(x[:S], positions[:S], torch.arange(S + 1, device="cuda"), torch.tensor(one, device="cuda"))
    ref = fp32_step(seen, layer.A, layer.B, scale, layer.q_weight, layer.k_weight, D, q_heads * D, x[:S], positions[:S],
                    [(i, i + 1, one[i]) for i in range(S)], dq[:S], dk[:S])
    far["served queries"], far["served keys"] = off(q1, ref[0]), off(k1, ref[1])
    for name, d in far.items():
        print(f"{name:16s} {d:.2e} from FP32")
    return far


if __name__ == "__main__":
    main()
