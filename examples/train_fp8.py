"""Trains a two-layer language-model head with the low-precision operators, and serves single tokens with the result.

    python examples/train_fp8.py [--steps 20] [--tokens 2048] [--features 1024] [--hidden 512] [--vocab 8192]

One step: the features and the first layer's weights are quantised to FP8 (with a scale per 128 elements, per 128 x 128 square), the layer's
output is their product; the second layer's cross entropy over the vocabulary and its gradient never hold the vocabulary's outputs as a whole;
the gradient of the first layer's output is quantised in both directions and gives the gradients of its weights and of the features.  The
master weights are FP32, updated by plain gradient descent.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2508_00441_amd import binding as oz, device  # noqa: E402

IGNORE = -100


def ceil(n: int, to: int) -> int:
    return -(-n // to) * to


class Quantised:
    """The E4M3 codes of a matrix (rows x k) and of its transpose, and their scales."""

    def __init__(self, rows: int, k: int, scaling: int):
        shared = oz.SCALE_BLOCK if scaling == oz.SCALE_BLOCKS else 1
        blocks = lambda n: -(-n // oz.SCALE_BLOCK)  # noqa: E731
        self.rows, self.k, self.scaling = rows, k, scaling
        self.Q = torch.empty((rows, ceil(k, 16)), dtype=torch.uint8, device="cuda")
        self.S = torch.empty((blocks(k), -(-rows // shared)), device="cuda")
        self.Qt = torch.empty((k, ceil(rows, 16)), dtype=torch.uint8, device="cuda")
        self.St = torch.empty((blocks(rows), -(-k // shared)), device="cuda")

    def take(self, X: torch.Tensor) -> "Quantised":
        oz.ozaki_quantise_fp8(self.rows, self.k, X, X.stride(0), oz.TYPES["f32" if X.dtype == torch.float32 else "bf16"], self.scaling, self.Q,
                              self.Q.shape[1], self.S, self.S.shape[1], self.Qt, self.Qt.shape[1], self.St, self.St.shape[1])
        return self


def product(m, n, k, A, Sa, B, Sb, scaling_b, D):
    oz.ozaki_gemm_fp8(m, n, k, A, A.shape[1], Sa, Sa.shape[1], B, B.shape[1], Sb, Sb.shape[1], scaling_b, D, D.shape[1],
                      oz.TYPES["f32" if D.dtype == torch.float32 else "bf16"])


class Head:
    def __init__(self, tokens: int, features: int, hidden: int, vocab: int, seed: int = 0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.tokens, self.features, self.hidden, self.vocab = tokens, features, hidden, vocab
        self.W1 = torch.randn((hidden, features), device="cuda", generator=gen) / features ** 0.5
        self.W2 = torch.randn((vocab, hidden), device="cuda", generator=gen) / hidden ** 0.5
        bf16 = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.x8, self.w8, self.g8 = (Quantised(tokens, features, oz.SCALE_VECTORS), Quantised(hidden, features, oz.SCALE_BLOCKS),
                                     Quantised(tokens, hidden, oz.SCALE_VECTORS))
        self.h, self.dh, self.dx = bf16(tokens, hidden), bf16(tokens, hidden), bf16(tokens, features)
        self.w2, self.dW2 = bf16(vocab, hidden), bf16(vocab, hidden)
        self.dW1 = torch.empty((hidden, features), device="cuda")
        self.loss, self.lse, self.dloss = (torch.empty((tokens,), device="cuda") for _ in range(3))
        need = [oz.ozaki_linear_loss_workspace_bytes(tokens, vocab, hidden, grad, False) for grad in (False, True)]
        need += [oz.ozaki_gemm_fp8_workspace_bytes(*s) for s in ((tokens, hidden, features), (tokens, features, hidden), (hidden, features, tokens),
                                                                 (1, hidden, features))]
        self.workspace = device.Workspace(max(need))
        self.requantise()

    def requantise(self):
        self.w8.take(self.W1)
        self.w2.copy_(self.W2)

    def forward(self, x, targets):
        """The mean loss of the tokens that count, as a tensor."""
        t, f, h, v = self.tokens, self.features, self.hidden, self.vocab
        self.x8.take(x)
        product(t, h, f, self.x8.Q, self.x8.S, self.w8.Q, self.w8.S, oz.SCALE_BLOCKS, self.h)
        oz.ozaki_linear_loss(t, v, h, self.h, h, self.w2, h, oz.TYPE_BF16, targets, IGNORE, self.loss, self.lse)
        counts = targets != IGNORE
        self.dloss.copy_(counts / counts.sum().clamp(min=1))
        return (self.loss * self.dloss).sum()

    def backward(self, targets):
        """dW2, dW1 and the gradient of the features, dx."""
        t, f, h, v = self.tokens, self.features, self.hidden, self.vocab
        oz.ozaki_linear_loss_grad(t, v, h, self.h, h, self.w2, h, oz.TYPE_BF16, targets, IGNORE, self.lse, self.dloss, self.dh, h, self.dW2, h)
        self.g8.take(self.dh)
        product(t, f, h, self.g8.Q, self.g8.S, self.w8.Qt, self.w8.St, oz.SCALE_BLOCKS, self.dx)
        product(h, f, t, self.g8.Qt, self.g8.St, self.x8.Qt, self.x8.St, oz.SCALE_VECTORS, self.dW1)

    def update(self, rate: float):
        self.W1.sub_(self.dW1, alpha=rate)
        self.W2.sub_(self.dW2, alpha=rate)
        self.requantise()

    def one_token(self, x):
        """One token: what the first layer makes of its features."""
        q = Quantised(1, self.features, oz.SCALE_VECTORS).take(x)
        h = torch.empty((1, self.hidden), dtype=torch.bfloat16, device="cuda")
        product(1, self.hidden, self.features, q.Q, q.S, self.w8.Q, self.w8.S, oz.SCALE_BLOCKS, h)
        return h

    def close(self):
        self.workspace.close()


def batch(tokens, features, vocab, seed):
    """Features and, for nine tokens of ten, targets that follow from them."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind = torch.randint(0, 64, (tokens,), device="cuda", generator=gen)
    means = torch.randn((64, features), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1234))
    x = (means[kind] + 0.5 * torch.randn((tokens, features), device="cuda", generator=gen)).to(torch.bfloat16)
    targets = kind * (vocab // 64)
    targets[torch.rand((tokens,), device="cuda", generator=gen) < 0.1] = IGNORE
    return x, targets


def train(steps=20, tokens=2048, features=1024, hidden=512, vocab=8192, rate=0.2, seed=0):
    head, losses = Head(tokens, features, hidden, vocab, seed), []
    for step in range(steps):
        x, targets = batch(tokens, features, vocab, step)
        losses.append(head.forward(x, targets))
        head.backward(targets)
        head.update(rate)
    return head, [float(v) for v in losses]


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("steps", 20), ("tokens", 2048), ("features", 1024), ("hidden", 512), ("vocab", 8192)):
        p.add_argument(f"--{name}", type=int, default=value)
    a = vars(p.parse_args())
    head, losses = train(**a)
    for i, v in enumerate(losses):
        print(f"step {i:3d}  loss {v:.4f}")
    assert oz.ozaki_last_device_status() == 0
    x, targets = batch(1, a["features"], a["vocab"], 99)
    h = head.one_token(x)
    loss, lse = torch.empty((64,), device="cuda"), torch.empty((64,), device="cuda")
    words = torch.arange(64, device="cuda") * (a["vocab"] // 64)
    oz.ozaki_linear_loss(64, a["vocab"], a["hidden"], h.expand(64, -1).contiguous(), a["hidden"], head.w2, a["hidden"], oz.TYPE_BF16, words, IGNORE, loss, lse)
    print(f"one token: word {int(words[loss.argmin()])}, target {int(targets[0])}")
    head.close()


if __name__ == "__main__":
    main()
