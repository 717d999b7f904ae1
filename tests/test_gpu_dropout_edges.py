"""The gradient through a dropped activation at widths whose last tile of columns is not full and whose tiles end inside a warp, with
guard bands around every result and a workspace of the queried size.  Tolerances are those of test_gpu_dropout.py."""
import numpy as np
import pytest
import torch

import paper_2302_06058_b200 as bm
from oracle import linear_oracle as LO
from oracle import residual_oracle as RO
from test_gpu_dropout import NUMBER, SEED, bf16_between, same

pytestmark = pytest.mark.gpu
PAD = 4096


def guarded(shape, dtype):
    """A view of `shape` inside a buffer of sevens, and the buffer."""
    n = int(np.prod(shape))
    b = torch.full((n + 2 * PAD,), 7.0, device="cuda").to(dtype)
    return b[PAD:PAD + n].view(shape), b


@pytest.mark.parametrize("act", [bm.ACT_NONE, bm.ACT_GELU, bm.ACT_SILU])
@pytest.mark.parametrize("C", [4128, 8224, 12320])
@pytest.mark.parametrize("T", [1, 3, 149, 700])
def test_tiles_that_are_not_full(T, C, act):
    rng = np.random.default_rng(T + C + act)
    X = torch.from_numpy(rng.standard_normal((T, C)) * 2).to(torch.bfloat16).cuda()
    q, s = torch.empty(T, C, dtype=torch.int8, device="cuda"), torch.empty(T, C // 32, dtype=torch.uint8, device="cuda")
    bm.bimask_ckpt_pack(X, T, C, q, s)
    z = LO.unpack(q.cpu().numpy(), s.cpu().numpy())
    d = bm.make_dropout(0.3, SEED, NUMBER)
    m = RO.multiplier(T, C, 0.3, SEED, NUMBER)
    dY = torch.from_numpy(rng.standard_normal((T, C))).to(torch.bfloat16).cuda()
    (dZ, b1), (db, b2) = guarded((T, C), torch.bfloat16), guarded((C,), torch.float32)
    ws, b3 = guarded((bm.bimask_linear_workspace_bytes(T, C, 32),), torch.uint8)
    zq, zs = (None, None) if act == bm.ACT_NONE else (q, s)
    bm.bimask_act_dropout_bwd(dY, zq, zs, act, d, T, C, dZ, db, ws, ws.numel())
    dy = dY.double().cpu().numpy()
    want, tol = dy * m * LO.slope(z, act), 5e-6 * np.abs(dy) * m
    assert bf16_between(dZ, want - tol, want + tol).all()
    assert (np.abs(db.double().cpu().numpy() - want.sum(0)) <= tol.sum(0) + (T + 8) * 2.0 ** -24 * np.abs(want).sum(0)).all()
    for b in (b1, b2, b3):
        assert bool((b[:PAD] == 7).all()) and bool((b[-PAD:] == 7).all())
    only = torch.empty_like(db)
    bm.bimask_act_dropout_bwd(dY, zq, zs, act, d, T, C, None, only, ws, ws.numel())
    bm.bimask_act_dropout_bwd(dY, zq, zs, act, d, T, C, dY, None, None, 0)                 # in place
    assert torch.equal(only, db) and same(dY, dZ)
