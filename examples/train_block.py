"""Trains a small language model of gated feed-forward blocks with the library's operators, and serves single tokens with the result.

    python examples/train_block.py [--steps 20] [--tokens 2048] [--width 512] [--hidden 1024] [--vocab 4096] [--blocks 2]

A block is a norm, a gated pair of linear layers and a linear layer back, whose result goes through a second norm and a gate into the sum that runs through
the model; what lies between two blocks is one call.  The output layer's cross entropy never holds the vocabulary's outputs as a whole.  A step computes
all gradients, scales them so that their norm over all tensors is at most one, and takes a step of plain gradient descent on 32-bit master weights.
"""
from __future__ import annotations

import argparse
import ctypes
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2508_00441_amd import binding as oz, device  # noqa: E402

IGNORE, EPS, BF16, SILU = -100, 1e-6, oz.TYPE_BF16, oz.ACTIVATION_SILU


class Model:
    def __init__(self, tokens: int, width: int, hidden: int, vocab: int, blocks: int, seed: int = 0):
        assert width % 8 == 0 and hidden % 8 == 0
        gen = torch.Generator(device="cuda").manual_seed(seed)
        randn = lambda *shape: torch.randn(shape, device="cuda", generator=gen)  # noqa: E731
        self.tokens, self.width, self.hidden, self.vocab, self.blocks = tokens, width, hidden, vocab, blocks
        # 32-bit master weights by name; matrices also in 16 bits, which the products read
        self.master = {"embedding": randn(vocab, width), "head": randn(vocab, width) / width ** 0.5, "pre0": torch.ones(width, device="cuda")}
        for i in range(blocks):
            self.master |= {f"gate_up{i}": randn(2 * hidden, width) / width ** 0.5, f"down{i}": randn(width, hidden) / hidden ** 0.5,
                            f"post{i}": torch.ones(width, device="cuda"), f"scale{i}": torch.full((1, width), 0.5, device="cuda"),
                            f"pre{i + 1}": torch.ones(width, device="cuda")}
        self.weights = {name: w.bfloat16() if w.shape[0] > 1 and w.dim() == 2 else w for name, w in self.master.items()}
        self.grads = {name: torch.zeros_like(w) for name, w in self.weights.items()}
        self.norm = torch.zeros((1,), device="cuda")
        # the clipping's table: the gradients lie in the same tensors at every step
        grads = list(self.grads.values())
        pointers = (ctypes.c_void_p * len(grads))(*[g.data_ptr() for g in grads])
        self.table = (len(grads), pointers, [g.numel() for g in grads], [oz.TYPE_F32 if g.dtype == torch.float32 else BF16 for g in grads])
        bf16 = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        # what the gradient needs of the forward call: the sum in front of and behind each block, the normed input, both factors and their product, the block's result
        self.sum = [bf16(tokens, width) for _ in range(blocks + 1)]
        self.normed = [bf16(tokens, width) for _ in range(blocks + 1)]
        self.g, self.u, self.h = ([bf16(tokens, hidden) for _ in range(blocks)] for _ in range(3))
        self.y = [bf16(tokens, width) for _ in range(blocks)]
        self.d_sum, self.d_normed, self.d_y, self.d_h = bf16(tokens, width), bf16(tokens, width), bf16(tokens, width), bf16(tokens, hidden)
        self.loss, self.lse, self.dloss = (torch.empty((tokens,), device="cuda") for _ in range(3))
        need = [oz.ozaki_gradient_norm_workspace_bytes(len(grads)), oz.ozaki_block_norm_workspace_bytes(tokens, width, tokens)]
        for m in (1, tokens):
            for grad in (False, True):
                need += [oz.ozaki_gated_linear_workspace_bytes(m, hidden, width, grad), oz.ozaki_linear_workspace_bytes(m, width, hidden, grad),
                         oz.ozaki_linear_loss_workspace_bytes(m, vocab, width, grad, False), oz.ozaki_linear_workspace_bytes(m, vocab, width, False)]
        need.append(oz.ozaki_block_norm_workspace_bytes(tokens, width, 0))
        self.workspace = device.Workspace(max(need))

    def _block(self, i, m, normed, total, g, u, h, y, total_out, normed_out):
        k, n, w = self.width, self.hidden, self.weights
        oz.ozaki_gated_linear(m, n, k, normed, k, w[f"gate_up{i}"], w[f"gate_up{i}"][n:], k, BF16, SILU, h, n, g, n if g is not None else 0, u, n if u is not None else 0)
        oz.ozaki_linear(m, k, n, h, n, w[f"down{i}"], n, BF16, None, oz.ACTIVATION_NONE, None, 0, y, k)
        oz.ozaki_block_norm(m, k, y, k, BF16, w[f"post{i}"], w[f"scale{i}"], m, 1.0, EPS, total, k, BF16, total_out, k, w[f"pre{i + 1}"], normed_out, k)

    def forward(self, words, targets):
        """The mean loss of the tokens that count, as a tensor."""
        t, k = self.tokens, self.width
        self.sum[0].copy_(self.weights["embedding"][words])
        oz.ozaki_block_norm(t, k, None, 0, BF16, None, None, 0, 1.0, EPS, self.sum[0], k, BF16, None, 0, self.weights["pre0"], self.normed[0], k)
        for i in range(self.blocks):
            self._block(i, t, self.normed[i], self.sum[i], self.g[i], self.u[i], self.h[i], self.y[i], self.sum[i + 1], self.normed[i + 1])
        oz.ozaki_linear_loss(t, self.vocab, k, self.normed[-1], k, self.weights["head"], k, BF16, targets, IGNORE, self.loss, self.lse)
        counts = targets != IGNORE
        self.dloss.copy_(counts / counts.sum().clamp(min=1))
        return (self.loss * self.dloss).sum()

    def backward(self, words, targets):
        """All gradients, into self.grads."""
        t, k, n, w, d = self.tokens, self.width, self.hidden, self.weights, self.grads
        oz.ozaki_linear_loss_grad(t, self.vocab, k, self.normed[-1], k, w["head"], k, BF16, targets, IGNORE, self.lse, self.dloss, self.d_normed, k, d["head"], k)
        d_sum = None                                                # (behind the last block the sum goes nowhere but through the norm)
        for i in reversed(range(self.blocks)):
            oz.ozaki_block_norm_grad(t, k, self.y[i], k, BF16, w[f"post{i}"], w[f"scale{i}"], t, 1.0, EPS, self.sum[i + 1], k, BF16, w[f"pre{i + 1}"], self.d_normed, k,
                                     d_sum, k, self.d_y, k, self.d_sum, k, d[f"post{i}"], d[f"scale{i}"], d[f"pre{i + 1}"])
            d_sum = self.d_sum
            oz.ozaki_linear_grad(t, k, n, self.h[i], n, w[f"down{i}"], n, BF16, oz.ACTIVATION_NONE, None, 0, self.d_y, k, self.d_h, n, d[f"down{i}"], n)
            both = d[f"gate_up{i}"]
            oz.ozaki_gated_linear_grad(t, n, k, self.normed[i], k, w[f"gate_up{i}"], w[f"gate_up{i}"][n:], k, BF16, SILU, self.g[i], n, self.u[i], n, self.d_h, n,
                                       self.d_normed, k, both, both[n:], k)
        oz.ozaki_block_norm_grad(t, k, None, 0, BF16, None, None, 0, 1.0, EPS, self.sum[0], k, BF16, w["pre0"], self.d_normed, k, d_sum, k, None, 0, self.d_sum, k,
                                 None, None, d["pre0"])
        d["embedding"].zero_().index_add_(0, words, self.d_sum)

    def update(self, rate: float):
        count, pointers, sizes, types = self.table
        oz.ozaki_clip_gradients(count, pointers, sizes, types, 1.0, 1.0, pointers, self.norm)
        for name, w in self.master.items():
            w.sub_(self.grads[name], alpha=rate)
            if self.weights[name] is not w:
                self.weights[name].copy_(w)

    def one_token(self, word):
        """What the output layer makes of one token: its outputs over the vocabulary."""
        k, n, w = self.width, self.hidden, self.weights
        bf16 = lambda m: torch.empty((1, m), dtype=torch.bfloat16, device="cuda")  # noqa: E731
        total, normed, h, y, z = w["embedding"][word].reshape(1, k).clone(), bf16(k), bf16(n), bf16(k), bf16(self.vocab)
        oz.ozaki_block_norm(1, k, None, 0, BF16, None, None, 0, 1.0, EPS, total, k, BF16, None, 0, w["pre0"], normed, k)
        for i in range(self.blocks):
            self._block(i, 1, normed, total, None, None, h, y, total, normed)
        oz.ozaki_linear(1, self.vocab, k, normed, k, w["head"], k, BF16, None, oz.ACTIVATION_NONE, None, 0, z, self.vocab)
        return z[0]

    def close(self):
        self.workspace.close()


def batch(tokens, vocab, seed):
    """Words, and for nine of ten the word that follows: a fixed permutation's."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    words = torch.randint(0, vocab, (tokens,), device="cuda", generator=gen)
    follows = torch.randperm(vocab, device="cuda", generator=torch.Generator(device="cuda").manual_seed(4321))
    targets = follows[words]
    targets[torch.rand((tokens,), device="cuda", generator=gen) < 0.1] = IGNORE
    return words, targets


def train(steps=20, tokens=2048, width=512, hidden=1024, vocab=4096, blocks=2, rate=2.0, seed=0):
    model, losses = Model(tokens, width, hidden, vocab, blocks, seed), []
    for step in range(steps):
        words, targets = batch(tokens, vocab, step)
        losses.append(model.forward(words, targets))
        model.backward(words, targets)
        model.update(rate)
    return model, [float(v) for v in losses]


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("steps", 20), ("tokens", 2048), ("width", 512), ("hidden", 1024), ("vocab", 4096), ("blocks", 2)):
        p.add_argument(f"--{name}", type=int, default=value)
    a = vars(p.parse_args())
    model, losses = train(**a)
    for i, v in enumerate(losses):
        print(f"step {i:3d}  loss {v:.4f}")
    assert oz.ozaki_last_device_status() == 0
    words, targets = batch(1, a["vocab"], 99)
    print(f"one token: word {int(model.one_token(words[0]).argmax())}, target {int(targets[0])}, norm of the last gradients {float(model.norm):.3f}")
    model.close()


if __name__ == "__main__":
    main()
