"""Activations at infinity, at the largest finite numbers and at NaN, on every kernel that applies them in the forward product
and in the restoring pass: minus infinity gives the limit 0, not the NaN of infinity times zero."""
import numpy as np
import pytest
import torch

import paper_2302_06058_b200 as bm

pytestmark = pytest.mark.gpu

ACTS = (bm.ACT_NONE, bm.ACT_RELU, bm.ACT_GELU, bm.ACT_GELU_TANH, bm.ACT_SILU)
Z = np.array([np.inf, -np.inf, np.nan, 3.0e38, -3.0e38, 200.0, -200.0, 0.0], np.float32)


def limits(act):
    if act == bm.ACT_NONE:
        return Z
    return np.where(np.isnan(Z), Z, np.maximum(Z, 0.0)).astype(np.float32)


# few tokens; pairs; one row tile; two row tiles per CTA; dense operand on pairs
@pytest.mark.parametrize("T,I,J,dense", [(4, 160, 64, False), (200, 288, 64, False), (200, 96, 64, False), (1040, 2080, 4096, False),
                                         (200, 288, 64, True)])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("act", ACTS)
def test_forward(act, residual, T, I, J, dense):
    """The product is zero, the bias is the pre-activation."""
    b = bm.alloc_layer_buffers(1, I, J, 1, dense=dense)
    N, M = (4, 8) if dense else (2, 4)
    bm.bimask_fwd_mask(torch.ones(I, J, device="cuda"), I, J, N, M, b["maskbits_f"], b["vals_f"], None if dense else b["meta_f"],
                       None if dense else b["hw_meta_f"])
    bias = np.resize(Z, I).astype(np.float32)
    X = torch.zeros(T, J, dtype=torch.bfloat16, device="cuda")
    R = torch.ones(T, I, dtype=torch.bfloat16, device="cuda") if residual else None
    Y = torch.empty(T, I, dtype=torch.bfloat16, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    bm.bimask_linear_fwd(X, b["vals_f"], None if dense else b["hw_meta_f"], torch.from_numpy(bias).cuda(), act, R, T, I, J, Y, None, None, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    want = torch.from_numpy(np.resize(limits(act), I) + np.float32(residual)).to(torch.bfloat16)
    got = Y.cpu()
    nan = torch.isnan(want)
    assert bool((torch.isnan(got) == nan).all())
    assert bool((got[:, ~nan] == want[~nan]).all())


@pytest.mark.parametrize("act", ACTS)
def test_restored_values(act):
    """A checkpoint whose values reach past fp32: +-127 * 2^127."""
    q = torch.zeros(2, 32, dtype=torch.int8, device="cuda")
    q[0], q[1] = 127, -127
    s = torch.full((2, 1), 254, dtype=torch.uint8, device="cuda")
    out = torch.empty(2, 32, dtype=torch.bfloat16, device="cuda")
    bm.bimask_ckpt_unpack(q, s, act, 2, 32, out)
    v = out.float().cpu().numpy()
    assert np.isposinf(v[0]).all() and (np.isneginf(v[1]).all() if act == bm.ACT_NONE else (v[1] == 0).all())
