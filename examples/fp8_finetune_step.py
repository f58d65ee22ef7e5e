"""A fine-tuning step whose frozen weights are in 8 bits and whose loss needs no logits.

One block: an up projection (frozen, 8 bits, with a LoRA adapter), a residual
connection with dropout, a down projection (frozen, 8 bits) and an output layer
(frozen), trained on the cross entropy of each token's label.  The gradient comes
from the loss's own call, goes through the 8-bit down projection, the dropout drawn
again, and ends in the adapter.

    python examples/fp8_finetune_step.py [--tokens M] [--features K] [--vocab N] [--steps S]
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2403_11366_amd as lora

BF16 = dict(dtype=torch.bfloat16, device="cuda")


class EightBitLayer:
    """A frozen weight [n, k] held in 8 bits, and what a step's calls on it need for up to
    `tokens` tokens."""

    def __init__(self, W: torch.Tensor, tokens: int):
        n, k = W.shape
        self.codes = torch.empty((n, (k + 127) // 128 * 128), dtype=torch.uint8, device=W.device)
        self.scales = torch.empty(lora.lora_fp8_scales_size(n, k), dtype=torch.uint8, device=W.device)
        lora.lora_fp8_quantize(W, self.codes, self.scales)
        self.n, self.k = n, k
        size = max(lora.lora_linear_fp8_fwd_workspace_size(tokens, n, k),
                   lora.lora_linear_fp8_bwd_workspace_size(tokens, n, k))
        self.workspace = torch.empty(size, dtype=torch.uint8, device=W.device)

    def values(self) -> torch.Tensor:
        """The weight that the codes stand for."""
        W = torch.empty((self.n, self.k), **BF16)
        lora.lora_fp8_dequantize(self.codes, self.scales, W)
        return W

    def forward(self, X: torch.Tensor) -> torch.Tensor:
        Y = torch.empty((X.shape[0], self.n), **BF16)
        lora.lora_linear_fp8_fwd(X, self.codes, self.scales, Y, self.workspace)
        return Y

    def backward(self, dY: torch.Tensor) -> torch.Tensor:
        dX = torch.empty((dY.shape[0], self.k), **BF16)
        lora.lora_linear_fp8_bwd(dY, self.codes, self.scales, dX, self.workspace)
        return dX


class Model:
    """hidden = X + dropout(W1 X + s B A X);  logits = W3 (W2 hidden).  Steps of up to
    `tokens` tokens."""

    def __init__(self, tokens: int, features: int, vocab: int, rank: int, p: float, seed: int):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        m, k, r = tokens, features, rank

        def weight(n, width, gain=1.0):
            return (torch.randn((n, width), generator=gen, device="cuda") * gain * width ** -0.5).to(torch.bfloat16)
        self.up, self.down = EightBitLayer(weight(k, k), m), EightBitLayer(weight(k, k), m)
        self.up_bf16 = self.up.values()       # what the adapter's own forward adds to
        self.head = weight(vocab, k, 2.0)
        self.A, self.B = weight(r, k), (torch.randn((k, r), generator=gen, device="cuda") * 0.02).to(torch.bfloat16)
        self.alpha, self.p, self.counter = float(2 * r), p, 0
        self.U = torch.empty((m, r), dtype=torch.float32, device="cuda")
        self.ws_lora = torch.empty(lora.lora_linear_bwd_workspace_size(m, k, k, r), dtype=torch.uint8, device="cuda")
        self.ws_loss = torch.empty(lora.lora_linear_xent_workspace_size(m, vocab, k, True, False), dtype=torch.uint8,
                                   device="cuda")
        self.loss = torch.empty(m, dtype=torch.float32, device="cuda")
        self.dA = torch.empty((r, k), dtype=torch.float32, device="cuda")
        self.dB = torch.empty((k, r), dtype=torch.float32, device="cuda")

    def step(self, X: torch.Tensor, labels: torch.Tensor, seed: int):
        """Losses of the tokens, and the adapter's gradients of their mean over labelled tokens."""
        m, k = X.shape
        U, loss = self.U[:m], self.loss[:m]
        Y, hidden = torch.empty((m, k), **BF16), torch.empty((m, k), **BF16)
        lora.lora_linear_fwd(X, self.up_bf16, self.A, self.B, Y, U, self.alpha)
        lora.lora_dropout(Y, hidden, seed, self.counter, self.p, residual=X)
        out = self.down.forward(hidden)
        labelled = (labels >= 0) & (labels < self.head.shape[0])
        dloss = labelled.float() / labelled.sum()
        dout = torch.empty((m, k), **BF16)
        lora.lora_linear_xent_step(out, self.head, labels, dloss, loss, dout, None, self.ws_loss)
        dhidden = self.down.backward(dout)
        dY, dX = torch.empty((m, k), **BF16), torch.empty((m, k), **BF16)
        lora.lora_dropout(dhidden, dY, seed, self.counter, self.p)     # the same elements as the forward's
        lora.lora_linear_bwd(dY, X, self.up_bf16, self.A, self.B, U, dX, self.dA, self.dB, self.ws_lora, self.alpha)
        self.counter += (m * k + 15) // 16
        return loss, self.dA, self.dB


def train(tokens: int = 512, features: int = 512, vocab: int = 8000, rank: int = 8, steps: int = 20, p: float = 0.05,
          lr: float = 0.5, seed: int = 0):
    """Mean losses of the steps on one batch."""
    model = Model(tokens, features, vocab, rank, p, seed)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    X = torch.randn((tokens, features), generator=gen, device="cuda").to(torch.bfloat16)
    labels = torch.randint(0, vocab, (tokens,), generator=gen, device="cuda", dtype=torch.int32)
    labels[: tokens // 8] = -100                                       # the prompt
    master = [model.A.float(), model.B.float()]
    losses = []
    for _ in range(steps):
        loss, dA, dB = model.step(X, labels, seed)
        losses.append(float(loss[tokens // 8:].mean()))
        for w, g, low in zip(master, (dA, dB), (model.A, model.B)):
            w -= lr * g
            low.copy_(w)
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--features", type=int, default=512)
    ap.add_argument("--vocab", type=int, default=8000)
    ap.add_argument("--steps", type=int, default=20)
    a = ap.parse_args()
    for i, x in enumerate(train(a.tokens, a.features, a.vocab, steps=a.steps)):
        print(f"step {i}: loss {x:.4f}")
