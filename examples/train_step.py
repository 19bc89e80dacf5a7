"""A data-parallel training step of a small language model, from its last hidden states to the chunk a rank sends.

    python examples/train_step.py [steps]

The model predicts the next token from the current one: an embedding, a mixing matrix and a head over the vocabulary.  PyTorch
differentiates the two layers in front; everything from the hidden states on runs in this library's kernels:

  cgx_head_loss, cgx_head_loss_grad   the loss over the vocabulary and its gradients, without the logits
  cgx_grad_clip                       (with no limit yet) the gradients of all layers, converted into one fused buffer
  cgx_quantize                        that buffer, compressed layer by layer: what the rank would send
  cgx_dequantize                      the gradient that every rank holds after the exchange (here there is one rank)
  cgx_grad_norm, cgx_grad_clip        its norm, and its clipping in place

The norm is that of the exchanged gradient, so all ranks clip by the same factor.  Clipping a rank's own gradients ahead of the exchange
would give each rank a factor of its own, and the step another direction.
"""
import math
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2111_08617_amd import binding as cgx  # noqa: E402

VOCAB, WIDTH, BATCH = 5003, 256, 1024
IGNORE = -100


class Model:
    """Binary32 embedding and mixing matrix, bfloat16 head: gradients of two types in one fused buffer."""

    def __init__(self, seed: int):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.embedding = (torch.randn(VOCAB, WIDTH, device="cuda", generator=g) * 0.5).requires_grad_()
        self.mix = (torch.randn(WIDTH, WIDTH, device="cuda", generator=g) / WIDTH ** 0.5).requires_grad_()
        self.head = torch.randn(VOCAB, WIDTH, device="cuda", generator=g) * 0.05          # kept in binary32, used in bfloat16
        self.layers = [self.embedding, self.mix, self.head]
        offsets = np.concatenate([[0], np.cumsum([p.numel() for p in self.layers])])
        self.plan = cgx.Plan(offsets, np.array([8, 8, 8], np.uint8), bucket=128, dt=cgx.F32)
        self.fused = torch.empty(self.plan.n, device="cuda")
        packed_bytes, meta_bytes = cgx.cgx_sizes(self.plan)
        self.packed = torch.empty(packed_bytes, dtype=torch.uint8, device="cuda")
        self.meta = torch.empty(meta_bytes // 4, device="cuda")
        # what the head and the norm need, kept over the steps
        self.workspace = torch.empty(cgx.cgx_head_workspace(BATCH, WIDTH, VOCAB, cgx.BF16, grad=True), dtype=torch.uint8, device="cuda")
        self.norm_workspace = torch.empty(cgx.cgx_grad_norm_workspace(), dtype=torch.uint8, device="cuda")
        self.loss, self.lse = torch.empty(BATCH, device="cuda"), torch.empty(BATCH, device="cuda")
        self.norm, self.zero = torch.empty(1, device="cuda"), torch.zeros(1, device="cuda")

    def gradients(self, tokens, targets):
        """(mean loss, gradients of the layers) of one batch; targets may hold IGNORE."""
        hidden = torch.tanh(self.embedding[tokens] @ self.mix).to(torch.bfloat16)
        head = self.head.to(torch.bfloat16)
        cgx.cgx_head_loss(hidden.detach(), head, targets, self.loss, self.lse, self.workspace, ignore=IGNORE)
        counted = (targets != IGNORE).sum().clamp(min=1)
        dloss = (1.0 / counted).expand(BATCH).contiguous()
        dhidden, dhead = torch.empty_like(hidden), torch.empty_like(head)
        cgx.cgx_head_loss_grad(hidden.detach(), head, targets, self.lse, dloss, dhidden, dhead, self.workspace, ignore=IGNORE)
        self.embedding.grad = self.mix.grad = None
        hidden.backward(dhidden)
        return self.loss.sum() / counted, [self.embedding.grad, self.mix.grad, dhead]

    def step(self, tokens, targets, seed: int, rate: float = 2.0, max_norm: float = 1.0):
        loss, grads = self.gradients(tokens, targets)
        cgx.cgx_grad_clip(grads, self.zero, math.inf, out=self.fused)
        cgx.cgx_quantize(self.fused, self.plan, seed, self.packed, self.meta)
        # (ranks would exchange their chunks here, and average them)
        cgx.cgx_dequantize(self.packed, self.meta, self.plan, cgx.F32, self.fused)
        cgx.cgx_grad_norm([self.fused], self.norm, self.norm_workspace)
        cgx.cgx_grad_clip([self.fused], self.norm, max_norm)
        with torch.no_grad():
            for p, lo, hi in zip(self.layers, self.plan.offsets[:-1], self.plan.offsets[1:]):
                p -= rate * self.fused[lo:hi].view_as(p)
        return loss


def batch(step: int):
    """Tokens, and the ones that follow them under a fixed permutation; a tenth of the places have no target."""
    g = torch.Generator(device="cuda").manual_seed(1000 + step)
    tokens = (torch.rand(BATCH, device="cuda", generator=g) ** 2 * 500).long()
    targets = (tokens * 7 + 3) % VOCAB
    targets[torch.rand(BATCH, device="cuda", generator=g) < 0.1] = IGNORE
    return tokens, targets


def main(steps: int = 60):
    model, losses = Model(seed=0), []
    for k in range(steps):
        loss = model.step(*batch(k), seed=k)
        losses.append(loss)
        if k % 10 == 0 or k == steps - 1:
            print(f"step {k:3d}  loss {float(loss):.4f}  gradient norm {float(model.norm):.4f}", flush=True)
    return [float(x) for x in losses]


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 60)
