"""The stack of examples/residual_blocks.py: junctions, dropout and sparse layers together, against the same network in plain fp64."""
import os
import sys

import numpy as np
import pytest
import torch

from oracle import linear_oracle as LO
from oracle import residual_oracle as RO

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def masked(layer):
    """Weights under the forward mask and under the backward mask, fp64."""
    def bits(t, cols):
        return np.unpackbits(t.cpu().numpy().view(np.uint8), axis=1, bitorder="little")[:, :cols].astype(np.float64)

    f = bits(layer.b["maskbits_f"], layer.J)
    b = np.empty_like(f)
    b[layer.b["perm"].cpu().numpy()] = bits(layer.b["maskbits_b"], layer.J)      # row k of the backward mask is row perm[k] of W
    W = layer.W.to(torch.bfloat16).double().cpu().numpy()
    return f * W, b * W


def f64(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("T,width,hidden,blocks,p,step", [(200, 128, 352, 2, 0.2, 0), (1, 64, 96, 1, 0.3, 5), (97, 160, 64, 3, 0.0, 1)])
def test_one_step_against_plain_fp64(T, width, hidden, blocks, p, step):
    """Output and every gradient.  The allowance is 4e-2 of a result's largest magnitude: per block half a dozen roundings to
    bf16 (2^-8 at most) and two to a checkpoint (1/254 of a block's largest value) are chained, and every block adds its own."""
    import residual_blocks
    stack = residual_blocks.Stack(T + 3, width, hidden, blocks, p, seed=7)
    g = torch.Generator(device="cuda").manual_seed(5)
    for b in stack.blocks:
        for layer in (b.fc1, b.fc2):
            layer.bias.normal_(generator=g)
    for j in stack.junctions:
        for k, v in j.params.items():
            v.add_(0.2 * torch.randn(width, generator=g, device="cuda"))
    stack.step.fill_(step)
    X = torch.randn(T, width, generator=g, device="cuda")
    dN = torch.randn(T, width, generator=g, device="cuda").to(torch.bfloat16)
    out = stack.forward(X).clone()
    stack.search(11)
    dn = f64(dN)
    dX = stack.backward(dN.clone())
    torch.cuda.synchronize()
    assert not any(stack.status())

    eps, x, n, kept = float(np.float32(1e-5)), f64(X), None, []
    for i, j in enumerate(stack.junctions):
        q = {k: f64(v) for k, v in j.params.items()}
        kw = dict(pre=RO.LAYER, eps_pre=eps, w_pre=q["w_pre"], b_pre=q["b_pre"])
        y = m = None
        if i > 0:
            block = stack.blocks[i - 1]
            (f1, b1), (f2, b2) = masked(block.fc1), masked(block.fc2)
            mh = RO.multiplier(T, hidden, p, 7, ((2 * i - 1) << 40) + step)
            m = RO.multiplier(T, width, p, 7, ((2 * i) << 40) + step)
            h, z = LO.linear(n, f1, f64(block.fc1.bias), LO.GELU, None)
            y, _ = LO.linear(h * mh, f2, f64(block.fc2.bias), LO.NONE, None)
            kept.append((n, z, h * mh, mh, b1, b2))
            kw.update(post=RO.RMS, eps_post=eps, w_post=q["w_post"], scale=q["scale"], m=m)
        o = RO.forward(x, y, **kw)
        x, n = o["xo"], o["n"]
        kept.append((o, y, kw))
    want, got = {"out": n}, {"out": out}
    dx = None
    for i in reversed(range(len(stack.junctions))):
        o, y, kw = kept.pop()
        j = stack.junctions[i]
        grads = RO.backward(dx, dn, o["xo"], y, o["stats_post"], o["stats_pre"], **{k: v for k, v in kw.items() if k not in ("eps_pre", "eps_post", "b_pre")})
        dx = grads["dx"]
        for k in j.grads:
            want[f"{k}{i}"], got[f"{k}{i}"] = grads[k], j.grads[k]
        if i > 0:
            nin, z, hd, mh, b1, b2 = kept.pop()
            block, dy = stack.blocks[i - 1], grads["dy"]
            dz, db1 = LO.act_bwd(dy @ b2 * mh, z, LO.GELU)
            want.update({f"db1{i}": db1, f"db2{i}": dy.sum(0), f"dW1{i}": dz.T @ nin, f"dW2{i}": dy.T @ hd})
            got.update({f"db1{i}": block.fc1.db, f"db2{i}": block.fc2.db, f"dW1{i}": block.fc1.b["dW"], f"dW2{i}": block.fc2.b["dW"]})
            dn = dz @ b1
    want["dX"], got["dX"] = dx, dX
    for k, w in want.items():
        d = np.abs(f64(got[k]) - w).max()
        assert d <= 4e-2 * np.abs(w).max(), (k, d, np.abs(w).max())


def test_training_runs():
    import residual_blocks
    losses, stack = residual_blocks.train(tokens=256, width=128, hidden=256, blocks=2, steps=6, search_every=3)
    assert all(np.isfinite(losses)) and not any(stack.status()) and int(stack.step.item()) == 6
    for j in stack.junctions:
        assert all(bool(torch.isfinite(v).all()) for v in j.params.values())
    with pytest.raises(ValueError, match="at most"):
        stack.forward(torch.zeros(257, 128, device="cuda"))
