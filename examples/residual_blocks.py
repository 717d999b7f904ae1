"""Training a stack of transformer MLP blocks with sparse weights and a residual stream, in this library's calls alone:

    x_0 = input,  n_0 = norm(x_0)
    y_i = W2 drop(gelu(W1 n_i + b1)) + b2                         (W1, W2 under the bi-directional 2:4 masks)
    x_i+1 = x_i + scale_i * drop(norm'_i(y_i)),  n_i+1 = norm_i+1(x_i+1)
    output = n of the last junction

A junction (norm after the block, dropout, residual scale, addition, norm before the next block) is one call, its gradient
another.  A block keeps two 8-bit checkpoints, of its input and of its pre-activation; hidden values and all dropout masks are
recomputed in the backward pass, the masks from the step's number in device memory.

    python examples/residual_blocks.py [--tokens 4096] [--width 1024] [--hidden 4096] [--blocks 4] [--steps 20] [--dropout 0.1]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2302_06058_b200 as bm  # noqa: E402
from mlp_block import SparseLinear  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32


def _empty(*shape, dtype=BF16):
    return torch.empty(*shape, dtype=dtype, device="cuda")


class Block:
    """y = W2 drop(gelu(W1 n + b1)) + b2; at most T tokens."""

    def __init__(self, T, width, hidden, generator, drop):
        self.width, self.hidden, self.drop = width, hidden, drop
        self.fc1, self.fc2 = SparseLinear(T, width, hidden, generator), SparseLinear(T, hidden, width, generator)
        self.Nq, self.Ns = _empty(T, width, dtype=torch.int8), _empty(T, width // 32, dtype=torch.uint8)
        self.Zq, self.Zs = _empty(T, hidden, dtype=torch.int8), _empty(T, hidden // 32, dtype=torch.uint8)

    def forward(self, n, H, y):
        T = n.shape[0]
        bm.bimask_ckpt_pack(n, T, self.width, self.Nq, self.Ns)
        self.fc1.forward(n, bm.ACT_GELU, None, H, self.Zq, self.Zs)
        bm.bimask_dropout(H, bm.TYPE_BF16, T, self.hidden, self.drop, H)
        self.fc2.forward(H, bm.ACT_NONE, None, y)

    def backward(self, dy, H, dH, dn):
        T, a, b = dy.shape[0], self.fc1, self.fc2
        for layer in (a, b):
            layer.backward_operand()
        bm.bimask_act_bwd(dy, None, None, bm.ACT_NONE, T, b.I, None, b.db, b.ws, b.ws.numel())
        b.input_gradient(dy, dH)
        bm.bimask_ckpt_unpack_dropout(self.Zq, self.Zs, bm.ACT_GELU, self.drop, T, self.hidden, H)
        bm.bimask_wgrad(dy, H, T, b.I, b.J, b.b["dW"], b.b["ws"], b.b["ws"].numel(), b.b["status_word"])
        bm.bimask_act_dropout_bwd(dH, self.Zq, self.Zs, bm.ACT_GELU, self.drop, T, self.hidden, dH, a.db, a.ws, a.ws.numel())
        a.input_gradient(dH, dn)
        bm.bimask_wgrad_ckpt(dH, self.Nq, self.Ns, T, a.I, a.J, a.b["dW"], a.ws, a.ws.numel(), a.b["status_word"])


class Junction:
    """x' = x + scale * drop(norm'(y)), n = norm(x'); without `join` the norm alone, n = norm(x)."""

    def __init__(self, T, width, drop, join=True):
        self.width, self.drop, self.join = width, drop, join
        self.params = {"w_pre": torch.ones(width, device="cuda"), "b_pre": torch.zeros(width, device="cuda")}
        if join:
            self.params.update(w_post=torch.ones(width, device="cuda"), scale=torch.full((width,), 0.5, device="cuda"))
        self.grads = {"d" + k: torch.zeros_like(v) for k, v in self.params.items()}
        # kept until the backward pass
        self.xo, self.y = _empty(T, width, dtype=F32), _empty(T, width)
        self.stats_pre, self.stats_post = _empty(T, 2, dtype=F32), _empty(T, 2, dtype=F32)
        self.ws = _empty(bm.bimask_residual_norm_workspace_bytes(T, width), dtype=torch.uint8)
        self.status_word = torch.zeros(1, dtype=torch.int32, device="cuda")

    def _args(self, T, **buffers):
        b = {**self.params, "stats_pre": self.stats_pre[:T], "xo": self.xo[:T], "status_word": self.status_word, **buffers}
        if self.join:
            b.update(y=self.y[:T], stats_post=self.stats_post[:T])
        return bm.make_residual_args(T, self.width, b, bm.TYPE_F32, bm.NORM_RMS if self.join else bm.NORM_NONE, bm.NORM_LAYER,
                                     drop=self.drop if self.join else None)

    def forward(self, x, n):
        bm.bimask_residual_norm_fwd(self._args(x.shape[0], x=x, n=n))
        return self.xo[:x.shape[0]]

    def backward(self, dxo, dn, dx, dy):
        bm.bimask_residual_norm_bwd(self._args(dn.shape[0], dxo=dxo, dn=dn, dx=dx, dy=dy if self.join else None, ws=self.ws, **self.grads))


class Stack:
    """`blocks` blocks on a residual stream of `width`; a batch has at most T tokens."""

    def __init__(self, T, width, hidden, blocks, dropout=0.1, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.T = T
        self.step = torch.zeros(1, dtype=torch.int64, device="cuda")           # moves every mask on
        # a stream number per place, far enough apart that no step's number reaches the next place's
        drops = [bm.make_dropout(dropout, seed, (k + 1) << 40, self.step) for k in range(2 * blocks)]
        self.blocks = [Block(T, width, hidden, g, drops[2 * i]) for i in range(blocks)]
        self.junctions = [Junction(T, width, None, join=False)] + [Junction(T, width, drops[2 * i + 1]) for i in range(blocks)]
        self.n, self.H, self.dH = _empty(T, width), _empty(T, hidden), _empty(T, hidden)
        self.dx, self.dy = _empty(T, width, dtype=F32), _empty(T, width)

    def forward(self, x):
        T = x.shape[0]
        if T > self.T:
            raise ValueError(f"{T} tokens in blocks for at most {self.T}")
        n = self.n[:T]
        x = self.junctions[0].forward(x, n)
        for block, junction in zip(self.blocks, self.junctions[1:]):
            block.forward(n, self.H[:T], junction.y[:T])
            x = junction.forward(x, n)
        return n

    def backward(self, dn):
        """Gradients of every parameter; returns that of the input.  dn is overwritten."""
        T = dn.shape[0]
        dx, dy, dxo = self.dx[:T], self.dy[:T], None
        for block, junction in zip(reversed(self.blocks), reversed(self.junctions)):
            junction.backward(dxo, dn, dx, dy)
            block.backward(dy, self.H[:T], self.dH[:T], dn)
            dxo = dx
        self.junctions[0].backward(dxo, dn, dx, None)
        return dx

    def search(self, seed):
        for i, block in enumerate(self.blocks):
            block.fc1.search(seed + 2 * i)
            block.fc2.search(seed + 2 * i + 1)

    def update(self, lr):
        for block in self.blocks:
            block.fc1.update(lr)
            block.fc2.update(lr)
        for junction in self.junctions:
            for k, v in junction.params.items():
                v.sub_(lr * junction.grads["d" + k])
        self.step.add_(1)

    def status(self):
        words = [layer.b["status_word"] for block in self.blocks for layer in (block.fc1, block.fc2)]
        return [int(word.item()) for word in words + [junction.status_word for junction in self.junctions]]


def train(tokens=4096, width=1024, hidden=4096, blocks=4, steps=20, dropout=0.1, lr=1.0, search_every=10, seed=0):
    """A few SGD steps towards a fixed random target; returns the losses (half the mean squared error) and the stack."""
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    x = torch.randn(tokens, width, generator=g, device="cuda")
    target = 0.5 * torch.tanh(x.roll(1, dims=1)) + 0.5 * x
    stack, losses = Stack(tokens, width, hidden, blocks, dropout, seed), []
    for t in range(1, steps + 1):
        err = stack.forward(x).float() - target
        losses.append(0.5 * err.square().mean())
        if t % search_every == 0:
            stack.search(seed + t)
        stack.backward((err / err.numel()).to(BF16))
        stack.update(lr)
    return [float(v) for v in losses], stack


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("tokens", 4096), ("width", 1024), ("hidden", 4096), ("blocks", 4), ("steps", 20)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--dropout", type=float, default=0.1)
    a = ap.parse_args()
    losses, stack = train(a.tokens, a.width, a.hidden, a.blocks, a.steps, a.dropout)
    for t, v in enumerate(losses, 1):
        print(f"step {t:3d}  loss {v:.5f}")
    assert not any(stack.status()), stack.status()


if __name__ == "__main__":
    main()
