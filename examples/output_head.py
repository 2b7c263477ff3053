"""One step of a language model's output head with the low-precision operators, as a user would chain them.

serving:   residual + update -> norm in 8 bits -> logits = 8-bit product with the head's weights -> log
           probabilities of the sampled tokens, entropy, alternatives
training:  the same logits against a teacher's top logits -> loss and gradient of the logits -> gradient cut
           for both products -> gradient of the hidden states (through the norm) and of the weights

Run:  python examples/output_head.py [--tokens T] [--hidden H] [--vocab V]
Prints, for each result, how far it is from the same step in FP32 without 8-bit rounding.
"""

from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1811_10751_b200 as g  # noqa: E402

E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2


class OutputHead:
    """Norm and output projection with 8-bit operands.  Weights are kept in BF16 and cut once per update, straight
    (forward) and transposed (gradient of the input); buffers are kept from step to step."""

    def __init__(self, weight: torch.Tensor, norm_weight: torch.Tensor, tokens: int, eps: float = 1e-5):
        V, H = weight.shape
        self.weight, self.norm_weight, self.eps = weight, norm_weight, eps
        self.w, self.w_scales = g.new_fp8(V, H, E4M3, 128)
        self.wT, self.wT_scales = g.new_fp8(H, V, E4M3, 128)
        self.cut_weights()
        dev = weight.device
        self.x, self.x_scales = g.new_fp8(tokens, H)
        self.y = torch.empty((tokens, H), dtype=torch.bfloat16, device=dev)
        self.rstd = torch.empty(tokens, device=dev)
        self.logits = torch.empty((tokens, V), dtype=torch.bfloat16, device=dev)
        self.dlogits = torch.empty_like(self.logits)
        self.d, self.d_scales = g.new_fp8(tokens, V, E5M2)
        self.dT, self.dT_scales = g.new_fp8(V, tokens, E5M2)
        self.xT, self.xT_scales = g.new_fp8(H, tokens)
        self.dy = torch.empty((tokens, H), dtype=torch.bfloat16, device=dev)
        self.workspace = torch.empty(min(tokens, g.GPD_RMSNORM_MAX_PARTS) * H, device=dev)

    def cut_weights(self):
        g.gpd_quantize_blocks(self.weight, q=self.w, scales=self.w_scales, qT=self.wT, scalesT=self.wT_scales, block_rows=128)

    def forward(self, update, residual):
        """logits [T, V] of residual + update; the sum is stored over the residual."""
        g.gpd_rmsnorm_quant(update, self.norm_weight, self.eps, residual=residual, residual_out=residual, y=self.y,
                            q=self.x, scales=self.x_scales, rstd=self.rstd)
        g.gpd_gemm_fp8(self.x, self.x_scales, self.w, self.w_scales, self.logits)
        return self.logits

    def score(self, tokens, alternatives: int = 8):
        """Log probabilities of `tokens`, entropies, and the most likely alternatives of every row of the last logits."""
        T, dev = self.logits.shape[0], self.logits.device
        logp, lse, entropy = (torch.empty(T, device=dev) for _ in range(3))
        ids = torch.empty((T, alternatives), dtype=torch.int32, device=dev)
        ids_logp = torch.empty((T, alternatives), device=dev)
        g.gpd_token_logprobs(self.logits, tokens, logp, lse, entropy=entropy, top_ids=ids, top_logprobs=ids_logp)
        return logp, entropy, ids, ids_logp

    def distill(self, hidden, teacher_ids, teacher_logits, weights, dweight, temperature: float = 2.0):
        """Loss per row; gradients of the hidden states (returned), of the norm's weight (returned) and of the projection
        (added to the FP32 buffer dweight).  `hidden`: what forward left in the residual."""
        T, H = hidden.shape
        loss = torch.empty(T, device=hidden.device)
        g.gpd_distill_topk(self.logits, teacher_ids, teacher_logits, weights, loss, dlogits=self.dlogits, temperature=temperature)
        g.gpd_quantize_blocks(self.dlogits, q=self.d, scales=self.d_scales, qT=self.dT, scalesT=self.dT_scales)
        g.gpd_quantize_blocks(self.y, qT=self.xT, scalesT=self.xT_scales)
        g.gpd_gemm_fp8(self.d, self.d_scales, self.wT, self.wT_scales, self.dy)
        g.gpd_gemm_fp8(self.dT, self.dT_scales, self.xT, self.xT_scales, dweight, accumulate=True)
        dhidden, dnorm = torch.empty_like(hidden), torch.empty(H, device=hidden.device)
        g.gpd_rmsnorm_backward(self.dy, hidden, self.norm_weight, self.rstd, dhidden, dnorm, self.workspace)
        return loss, dhidden, dnorm


def fp32_step(weight, norm_weight, update, residual, teacher_ids, teacher_logits, weights, temperature, eps=1e-5):
    """The same step by automatic differentiation in FP32."""
    W, n = weight.float().requires_grad_(), norm_weight.float().requires_grad_()
    h = (update.float() + residual.float()).requires_grad_()
    logits = (h * torch.rsqrt(h.square().mean(1, keepdim=True) + eps) * n) @ W.t()
    logp = torch.log_softmax(logits / temperature, 1).gather(1, teacher_ids.long())
    logq = torch.log_softmax(teacher_logits / temperature, 1)
    loss = (logq.exp() * (logq - logp)).sum(1) * weights * temperature ** 2
    loss.sum().backward()
    return logits.detach(), loss.detach(), h.grad, n.grad, W.grad


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--vocab", type=int, default=8000)
    a = ap.parse_args(argv)
    gen = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    weight, norm_weight = (rand(a.vocab, a.hidden) * 2 / a.hidden ** 0.5).bfloat16(), (1 + 0.1 * rand(a.hidden)).bfloat16()
    update, residual = rand(a.tokens, a.hidden).bfloat16(), rand(a.tokens, a.hidden).bfloat16()
    teacher = torch.topk(rand(a.tokens, a.vocab) * 3, 20, dim=1)
    teacher_ids, teacher_logits = teacher.indices.int(), teacher.values.contiguous()
    weights = torch.full((a.tokens,), 1.0 / a.tokens, device="cuda")

    head = OutputHead(weight, norm_weight, a.tokens)
    before = residual.clone()
    logits = head.forward(update, residual)
    tokens = torch.randint(0, a.vocab, (a.tokens,), device="cuda", generator=gen)
    logp, entropy, ids, ids_logp = head.score(tokens)
    dweight = torch.zeros((a.vocab, a.hidden), device="cuda")
    loss, dhidden, dnorm = head.distill(residual, teacher_ids, teacher_logits, weights, dweight)
    assert g.gpd_device_status() == 0

    ref = fp32_step(weight, norm_weight, update, before, teacher_ids, teacher_logits, weights, 2.0)
    rlogp = torch.log_softmax(ref[0], 1)
    off = lambda x, y: float((x.float() - y).norm() / y.norm())  # noqa: E731
    far = {"logits": off(logits, ref[0]), "log probabilities": off(logp, rlogp.gather(1, tokens[:, None])[:, 0]),
           "entropy": off(entropy, -(rlogp.exp() * rlogp).sum(1)), "loss": off(loss, ref[1]), "d hidden": off(dhidden, ref[2]),
           "d norm weight": off(dnorm, ref[3]), "d weight": off(dweight, ref[4])}
    for name, d in far.items():
        print(f"{name:18s} {d:.2e} from FP32")
    print("alternatives of row 0:", ids[0].tolist(), [round(v, 3) for v in ids_logp[0].tolist()])
    return far


if __name__ == "__main__":
    main()
