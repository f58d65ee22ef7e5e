"""Distillation of an output layer into a LoRA adapter.

The teacher is a fine-tuned output layer, its adapter merged into the weight and
the weight held in microscaled 4-bit floating point.  For every batch it forms
its logits, of which the largest of each token are kept; the student, the same
layer without the fine-tuning and with a fresh adapter, takes a step on the
distillation loss against that list and the labels.  At the end the student's
adapter is merged and put into 4 bits too, and both score one token.

    python examples/distill_step.py [--tokens M] [--features K] [--vocab N] [--steps S]
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2403_11366_amd as lora


class FourBitLayer:
    """A weight [n, k] held in 4 bits, and what its forward needs."""

    def __init__(self, W: torch.Tensor, tokens: int):
        n, k = W.shape
        self.codes = torch.empty((n, (k + 255) // 256 * 128), dtype=torch.uint8, device=W.device)
        self.scales = torch.empty(lora.lora_mx4_scales_size(n, k), dtype=torch.uint8, device=W.device)
        lora.lora_mx4_quantize(W, self.codes, self.scales)
        self.n, self.k = n, k
        self.workspace = torch.empty(lora.lora_linear_mx4_fwd_workspace_size(tokens, n, k), dtype=torch.uint8,
                                     device=W.device)

    def __call__(self, X: torch.Tensor) -> torch.Tensor:
        Y = torch.empty((X.shape[0], self.n), dtype=torch.bfloat16, device=X.device)
        lora.lora_linear_mx4_fwd(X, self.codes, self.scales, Y, self.workspace)
        return Y


def score(logits: torch.Tensor, tokens: torch.Tensor, top: int):
    """(log probability of each row's token, entropy, top ids, their log probabilities)"""
    rows, vocab = logits.shape
    like = dict(device=logits.device)
    out = (torch.empty(rows, **like), torch.empty(rows, **like), torch.empty((rows, top), dtype=torch.int32, **like),
           torch.empty((rows, top), **like))
    workspace = torch.empty(lora.lora_token_logprobs_workspace_size(rows, vocab, top), dtype=torch.uint8, **like)
    lora.lora_token_logprobs(logits, tokens, *out, workspace)
    return out


class Adapter:
    """A [r, k] and B [n, r] in bf16 over fp32 masters, with Adam's moments."""

    def __init__(self, n: int, k: int, r: int, generator: torch.Generator, lr: float):
        A = torch.randn((r, k), generator=generator, device="cuda") / k ** 0.5
        self.master = [A, torch.zeros((n, r), device="cuda")]
        self.first = [torch.zeros_like(p) for p in self.master]
        self.second = [torch.zeros_like(p) for p in self.master]
        self.A, self.B = (p.to(torch.bfloat16) for p in self.master)
        self.lr, self.t = lr, 0

    def update(self, grads) -> None:
        self.t += 1
        for p, g, m1, m2, low in zip(self.master, grads, self.first, self.second, (self.A, self.B)):
            m1.lerp_(g, 0.1)
            m2.lerp_(g * g, 0.01)
            p -= self.lr * (m1 / (1 - 0.9 ** self.t)) / ((m2 / (1 - 0.99 ** self.t)).sqrt() + 1e-8)
            low.copy_(p)


def train(tokens: int = 1024, features: int = 1024, vocab: int = 32000, rank: int = 16, top: int = 32, steps: int = 30,
          temperature: float = 2.0, soft_weight: float = 0.75, lr: float = 2e-2, seed: int = 0):
    """Losses of the steps, and the log probability of one token by teacher and student."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    m, n, k, r, alpha = tokens, vocab, features, rank, float(rank)
    bf16 = dict(dtype=torch.bfloat16, device="cuda")
    W = (torch.randn((n, k), generator=gen, device="cuda") / k ** 0.5).to(torch.bfloat16)
    # the teacher: W + B A, merged and put into 4 bits
    At = (torch.randn((r, k), generator=gen, device="cuda") / k ** 0.5).to(torch.bfloat16)
    Bt = torch.randn((n, r), generator=gen, device="cuda").to(torch.bfloat16)
    merged = torch.empty_like(W)
    lora.lora_linear_merge(W, At, Bt, merged, alpha)
    teacher = FourBitLayer(merged, m)

    student = Adapter(n, k, r, gen, lr)
    Y, dX, U = torch.empty((m, n), **bf16), torch.empty((m, k), **bf16), torch.empty((m, r), device="cuda")
    dA, dB = torch.empty((r, k), device="cuda"), torch.empty((n, r), device="cuda")
    workspace = torch.empty(lora.lora_linear_bwd_workspace_size(m, n, k, r), dtype=torch.uint8, device="cuda")
    loss, dloss = torch.empty(m, device="cuda"), torch.full((m,), 1.0 / m, device="cuda")
    losses = []
    for _ in range(steps):
        X = torch.randn((m, k), generator=gen, device="cuda").to(torch.bfloat16)
        logits = teacher(X)
        labels = logits.argmax(dim=1).to(torch.int32)
        # (log probabilities are logits less a row's constant, which the loss does not see)
        _, _, ids, top_logp = score(logits, labels, top)
        lora.lora_linear_fwd(X, W, student.A, student.B, Y, U, alpha)
        lora.lora_distill_step(Y, ids, top_logp, labels, dloss, loss, Y, temperature=temperature,
                               soft_weight=soft_weight)        # the gradient takes the logits' place
        lora.lora_linear_bwd(Y, X, W, student.A, student.B, U, dX, dA, dB, workspace, alpha)
        student.update((dA, dB))
        losses.append(float(loss.mean()))

    lora.lora_linear_merge(W, student.A, student.B, merged, alpha)
    X = torch.randn((1, k), generator=gen, device="cuda").to(torch.bfloat16)
    one = teacher(X)
    token = one.argmax(dim=1).to(torch.int32)
    return losses, [float(score(z, token, 1)[0]) for z in (one, FourBitLayer(merged, 1)(X), FourBitLayer(W, 1)(X))]


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--tokens", type=int, default=1024)
    p.add_argument("--features", type=int, default=1024)
    p.add_argument("--vocab", type=int, default=32000)
    p.add_argument("--steps", type=int, default=30)
    a = p.parse_args()
    losses, scores = train(a.tokens, a.features, a.vocab, steps=a.steps)
    for i, x in enumerate(losses):
        print(f"step {i:3d}  loss {x:.4f}")
    print("log probability of the teacher's token: teacher %.3f, student %.3f, without the adapter %.3f" % tuple(scores))


if __name__ == "__main__":
    main()
