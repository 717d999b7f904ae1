"""The persistent kernels of bimask_linear_fwd over several tiles per CTA pair: barrier phases that wrap across tiles, the
residual of the next tile loaded ahead, accumulators handed back.  Residual and checkpoint together; sums, bias and residual
are small multiples of 1/2, so that every byte must be equal."""
import numpy as np
import pytest
import torch

import paper_2302_06058_b200 as bm
from test_gpu_linear import bf, cuda, operand, pack_fast, run_linear

pytestmark = pytest.mark.gpu

PAIRS = 74


def tiles_at_least(T, I, rows):
    """No token tile is wider than 256."""
    return (I + rows - 1) // rows * ((T + 255) // 256)


# kernel (2 pairs, 3 two row tiles each), tokens x rows x reduction, pattern
@pytest.mark.parametrize("kernel,T,I,J,N,M", [(3, 11521, 2080, 4096, 2, 4), (3, 4353, 6176, 4128, 2, 4), (2, 28673, 416, 160, 2, 4),
                                              (2, 11601, 1184, 96, 1, 4), (2, 28673, 288, 96, 4, 8), (2, 11601, 1184, 160, 4, 8)])
def test_exact_over_several_tiles_per_pair(kernel, T, I, J, N, M):
    assert bm.bimask_debug_linear_plan(T, I, J, N > 2)[0] == kernel
    assert tiles_at_least(T, I, 512 if kernel == 3 else 256) >= 3 * PAIRS
    rng = np.random.default_rng(T + I + J)
    vals, hw, Wm = operand(rng.integers(-2, 3, (I, J)).astype(np.float64), N, M)
    X, _ = bf(rng.integers(-2, 3, (T, J)))
    bias = rng.integers(-9, 10, I) * 0.5
    R, r = bf(rng.integers(-4, 5, (T, I)) * 0.5)
    z = (X.double() @ cuda(Wm).t() + cuda(bias)).cpu().numpy()
    q0, s0 = pack_fast(z)
    want = torch.from_numpy(np.maximum(z, 0.0) + r).float().to(torch.bfloat16)
    for use_r, use_c in ((True, True), (True, False), (False, True)):
        Y, q, s = run_linear(vals, hw, X, cuda(bias, torch.float32), bm.ACT_RELU, R if use_r else None, T, I, J, use_c)
        assert torch.equal(Y.cpu(), want if use_r else torch.from_numpy(np.maximum(z, 0.0)).float().to(torch.bfloat16)), (use_r, use_c)
        if use_c:
            assert np.array_equal(s.cpu().numpy(), s0) and np.array_equal(q.cpu().numpy(), q0), (use_r, use_c)
    both = R.clone()                                         # the residual in place
    Y, _, _ = run_linear(vals, hw, X, cuda(bias, torch.float32), bm.ACT_RELU, both, T, I, J, False, Y=both)
    assert torch.equal(Y.cpu(), want)


@pytest.mark.parametrize("T,I,J", [(9, 96, 160), (300, 288, 160)])
def test_relu_forward_and_backward_together(T, I, J):
    """The gradient through a ReLU layer goes by its checkpoint: channels whose pre-activation rounds to the byte 0 get none, active
    ones among them; all others get what the exact pre-activation says."""
    rng = np.random.default_rng(T)
    vals, hw, Wm = operand(rng.standard_normal((I, J)), 2, 4)
    X, x = bf(rng.standard_normal((T, J)))
    bias = rng.standard_normal(I).astype(np.float32)
    dY, dy = bf(rng.standard_normal((T, I)))
    Y, q, s = run_linear(vals, hw, X, cuda(bias), bm.ACT_RELU, None, T, I, J, True)
    dZ, db = torch.empty_like(dY), torch.empty(I, device="cuda")
    ws = torch.empty(bm.bimask_linear_workspace_bytes(T, I, 32), dtype=torch.uint8, device="cuda")
    bm.bimask_act_bwd(dY, q, s, bm.ACT_RELU, T, I, dZ, db, ws, ws.numel())
    z = x @ Wm.T + bias
    p = np.repeat(np.exp2(s.cpu().numpy().astype(np.float64) - 127.0), 32, axis=1)
    acc = (J / 16 + 32) * 2.0 ** -23 * (np.abs(x) @ np.abs(Wm).T + np.abs(bias))
    got = dZ.double().cpu().numpy()
    lost = (z > 0) & (z < p / 2 - acc)
    sure = (z < 0) | (z > p / 2 + acc)
    assert np.array_equal(got[lost], np.zeros(lost.sum())) and lost.any()
    assert np.array_equal(got[sure], np.where(z > 0, dy, 0.0)[sure])
    active = (Y.float() > 0).cpu().numpy()
    assert lost.sum() < 0.03 * active.sum()                  # about one active channel in a hundred on normal pre-activations
    want = got.sum(0)
    assert (np.abs(db.double().cpu().numpy() - want) <= (T + 64) * 2.0 ** -24 * np.abs(got).sum(0)).all()
