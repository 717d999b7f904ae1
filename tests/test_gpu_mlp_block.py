"""The MLP block of examples/mlp_block.py: its calls together, against the same block written in plain fp64."""
import os
import sys

import numpy as np
import pytest
import torch

from oracle import linear_oracle as LO

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def masks(layer):
    def bits(t, cols):
        return np.unpackbits(t.cpu().numpy().view(np.uint8), axis=1, bitorder="little")[:, :cols].astype(np.float64)

    f = bits(layer.b["maskbits_f"], layer.J)
    b = np.empty_like(f)
    b[layer.b["perm"].cpu().numpy()] = bits(layer.b["maskbits_b"], layer.J)      # row k of the backward mask is row perm[k] of W
    W = layer.W.to(torch.bfloat16).double().cpu().numpy()
    return f * W, b * W


@pytest.mark.parametrize("T,width,hidden", [(300, 128, 352), (1, 64, 96), (97, 160, 64)])
def test_one_step_against_plain_fp64(T, width, hidden):
    """Forward values, both checkpoints and every gradient.  The allowance is 2e-2 of a result's largest magnitude: a few
    roundings to bf16 (2^-8) and to a checkpoint (1/254 of a block's largest value) are chained on the way."""
    import mlp_block
    block = mlp_block.SparseMLP(T, width, hidden, seed=3)
    for layer in (block.fc1, block.fc2):
        layer.bias.normal_(generator=torch.Generator(device="cuda").manual_seed(5))
    g = torch.Generator(device="cuda").manual_seed(9)
    X = torch.randn(T, width, generator=g, device="cuda").to(torch.bfloat16)
    dY = torch.randn(T, width, generator=g, device="cuda").to(torch.bfloat16)
    Y = block.forward(X).clone()
    block.search(11)
    dX = block.backward(dY).clone()
    torch.cuda.synchronize()
    assert int(block.fc1.b["status_word"].item()) == 0 and int(block.fc2.b["status_word"].item()) == 0

    x, dy = X.double().cpu().numpy(), dY.double().cpu().numpy()
    (f1, b1), (f2, b2) = masks(block.fc1), masks(block.fc2)
    c1, c2 = (layer.bias.double().cpu().numpy() for layer in (block.fc1, block.fc2))
    h, z = LO.linear(x, f1, c1, LO.GELU, None)
    y, _ = LO.linear(h, f2, c2, LO.NONE, x)
    dz, db1 = LO.act_bwd(dy @ b2, z, LO.GELU)
    want = {"Y": y, "dX": dz @ b1 + dy, "db1": db1, "db2": dy.sum(0), "dW1": dz.T @ x, "dW2": dy.T @ h}
    got = {"Y": Y, "dX": dX, "db1": block.fc1.db, "db2": block.fc2.db, "dW1": block.fc1.b["dW"], "dW2": block.fc2.b["dW"]}
    for k, w in want.items():
        d = np.abs(got[k].double().cpu().numpy() - w).max()
        assert d <= 2e-2 * np.abs(w).max(), (k, d, np.abs(w).max())
    kept = LO.unpack(block.Zq.cpu().numpy(), block.Zs.cpu().numpy())
    top = np.repeat(np.abs(z.reshape(T, -1, 32)).max(-1), 32, axis=1)
    assert (np.abs(kept - z) <= top / 127 + 1e-4).all()


def test_a_few_steps_lower_the_loss():
    import mlp_block
    losses, block = mlp_block.train(tokens=512, width=128, hidden=512, steps=30, search_every=10)
    assert all(np.isfinite(losses)) and losses[-1] < 0.8 * losses[0], losses
    assert block.kept_bytes() == 512 * (128 + 512) * 33 // 32
