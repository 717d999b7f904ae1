"""Training a transformer MLP block with sparse weights, in this library's calls alone:

    Y = X + W2 gelu(W1 X + b1) + b2        (W1, W2 under the bi-directional 2:4 masks)

What the block keeps from the forward to the backward pass are two 8-bit checkpoints, its input and its pre-activation:
33 bytes for every 64 of bf16, and the activated values are recomputed instead of kept.

    python examples/mlp_block.py [--tokens 4096] [--width 1024] [--hidden 4096] [--steps 20]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2302_06058_b200 as bm  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32


def _empty(*shape, dtype=BF16):
    return torch.empty(*shape, dtype=dtype, device="cuda")


class SparseLinear:
    """Weights, bias and buffers of one layer: `inputs` -> `outputs`, at most T tokens."""

    def __init__(self, T, inputs, outputs, generator, P=32):
        self.T, self.I, self.J, self.P = T, outputs, inputs, P
        self.b = bm.alloc_layer_buffers(T, outputs, inputs, P)
        self.W = torch.randn(outputs, inputs, generator=generator, device="cuda") * (2.0 / inputs) ** 0.5
        self.bias = torch.zeros(outputs, device="cuda")
        self.momentum = torch.zeros_like(self.W)
        self.db = _empty(outputs, dtype=F32)
        self.ws = _empty(bm.bimask_linear_workspace_bytes(T, outputs, inputs), dtype=torch.uint8)
        b = self.b
        bm.bimask_fwd_mask(self.W, self.I, self.J, 2, 4, b["maskbits_f"], b["vals_f"], b["meta_f"], b["hw_meta_f"])

    def search(self, seed):
        """A new row permutation (every so many iterations) and the backward operand of the current weights."""
        b = self.b
        bm.bimask_perm_search(b["maskbits_f"], self.I, self.J, 2, 4, self.P, seed, None, b["perm"], b["best_idx"], b["counts"], b["ws"],
                              b["ws"].numel())

    def backward_operand(self):
        b = self.b
        bm.bimask_bwd_mask(self.W, b["maskbits_f"], b["perm"], self.I, self.J, 2, 4, b["maskbits_b"], b["vals_b"], b["meta_b"], b["hw_meta_b"])

    def forward(self, X, act, residual, Y, Zq=None, Zs=None):
        b = self.b
        bm.bimask_linear_fwd(X, b["vals_f"], b["hw_meta_f"], self.bias, act, residual, X.shape[0], self.I, self.J, Y, Zq, Zs, b["status_word"])

    def input_gradient(self, dZ, dX):
        b = self.b
        bm.bimask_spmm_dgrad(dZ, b["perm"], b["vals_b"], b["hw_meta_b"], dZ.shape[0], self.I, self.J, dX, b["ws"], b["ws"].numel(),
                             b["status_word"])

    def update(self, lr):
        """SGD on the dense weights (straight-through) with the next forward mask, and on the bias."""
        b = self.b
        bm.bimask_sgd_fwd_mask(self.W, b["dW"], self.momentum, self.I, self.J, 2, 4, lr, 0.9, 0.0, b["maskbits_f"], b["vals_f"], b["meta_f"],
                               b["hw_meta_f"])
        self.bias.sub_(lr * self.db)


class SparseMLP:
    """The block; a batch has at most T tokens."""

    def __init__(self, T, width, hidden, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.T, self.width, self.hidden = T, width, hidden
        self.fc1, self.fc2 = SparseLinear(T, width, hidden, g), SparseLinear(T, hidden, width, g)
        # kept until the backward pass
        self.Xq, self.Xs = _empty(T, width, dtype=torch.int8), _empty(T, width // 32, dtype=torch.uint8)
        self.Zq, self.Zs = _empty(T, hidden, dtype=torch.int8), _empty(T, hidden // 32, dtype=torch.uint8)
        # used and given back within a pass
        self.H, self.Y, self.dH, self.dX = _empty(T, hidden), _empty(T, width), _empty(T, hidden), _empty(T, width)

    def kept_bytes(self):
        return sum(t.numel() for t in (self.Xq, self.Xs, self.Zq, self.Zs))

    def forward(self, X):
        T = X.shape[0]                                    # this batch's tokens: the first T rows of every buffer
        if T > self.T:
            raise ValueError(f"{T} tokens in a block for at most {self.T}")
        bm.bimask_ckpt_pack(X, T, self.width, self.Xq, self.Xs)
        self.fc1.forward(X, bm.ACT_GELU, None, self.H[:T], self.Zq, self.Zs)
        self.fc2.forward(self.H[:T], bm.ACT_NONE, X, self.Y[:T])
        return self.Y[:T]

    def backward(self, dY):
        T, a, b = dY.shape[0], self.fc1, self.fc2
        H, dH, dX = self.H[:T], self.dH[:T], self.dX[:T]
        for layer in (a, b):
            layer.backward_operand()
        # second layer: bias, input and weight gradient, its input recomputed from the pre-activation's checkpoint
        bm.bimask_act_bwd(dY, None, None, bm.ACT_NONE, T, b.I, None, b.db, b.ws, b.ws.numel())
        b.input_gradient(dY, dH)
        bm.bimask_ckpt_unpack(self.Zq, self.Zs, bm.ACT_GELU, T, self.hidden, H)
        bm.bimask_wgrad(dY, H, T, b.I, b.J, b.b["dW"], b.b["ws"], b.b["ws"].numel(), b.b["status_word"])
        # through the activation (in place), then the first layer
        bm.bimask_act_bwd(dH, self.Zq, self.Zs, bm.ACT_GELU, T, a.I, dH, a.db, a.ws, a.ws.numel())
        a.input_gradient(dH, dX)
        bm.bimask_wgrad_ckpt(dH, self.Xq, self.Xs, T, a.I, a.J, a.b["dW"], a.ws, a.ws.numel(), a.b["status_word"])
        return dX.add_(dY)                                # the residual's gradient is dY itself

    def search(self, seed):
        self.fc1.search(seed)
        self.fc2.search(seed + 1)

    def update(self, lr):
        self.fc1.update(lr)
        self.fc2.update(lr)


def train(tokens=4096, width=1024, hidden=4096, steps=20, lr=1.0, search_every=10, seed=0):
    """A few SGD steps towards a fixed random target; returns the losses (half the mean squared error) and the block."""
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    X = torch.randn(tokens, width, generator=g, device="cuda").to(BF16)
    target = (X.float() + 0.5 * torch.tanh(X.float().roll(1, dims=1))).to(BF16)
    block, losses = SparseMLP(tokens, width, hidden, seed), []
    for t in range(1, steps + 1):
        Y = block.forward(X)
        err = Y.float() - target.float()
        losses.append(0.5 * err.square().mean())
        if t % search_every == 0:
            block.search(seed + t)
        block.backward((err / err.numel()).to(BF16))
        block.update(lr)
    return [float(v) for v in losses], block


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("tokens", 4096), ("width", 1024), ("hidden", 4096), ("steps", 20)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    losses, block = train(a.tokens, a.width, a.hidden, a.steps)
    for t, v in enumerate(losses, 1):
        print(f"step {t:3d}  loss {v:.5f}")
    bf16 = 2 * a.tokens * (a.width + a.hidden)
    print(f"kept for the backward pass: {block.kept_bytes() / 2**20:.1f} MiB (bf16 input and pre-activation: {bf16 / 2**20:.1f} MiB)")
    status = [int(layer.b["status_word"].item()) for layer in (block.fc1, block.fc2)]
    assert status == [0, 0], status


if __name__ == "__main__":
    main()
