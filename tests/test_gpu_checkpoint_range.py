"""Checkpoints at the ends of the range: no finite value may come back infinite, small ones keep the documented error."""
import numpy as np
import pytest
import torch

import paper_2302_06058_b200 as bm
from oracle import linear_oracle as LO

pytestmark = pytest.mark.gpu

TOP = 127.0 * 2.0 ** 121                                     # the largest magnitude that a checkpoint holds
MAX = 255.0 * 2.0 ** 120                                     # the largest finite bf16


def test_pack_and_restore_at_the_largest_values():
    C = 64
    x = np.zeros((6, C))
    x[0, 3], x[1, 40], x[2, 0], x[3, 63], x[4, 5] = MAX, -MAX, TOP, -TOP, MAX
    x[4, 6] = 1.0                                            # a small value beside the largest one
    x[5, :32] = np.linspace(-TOP, TOP, 32)
    X = torch.from_numpy(x).float().to(torch.bfloat16).cuda()
    x = X.double().cpu().numpy()
    q, s = torch.empty(6, C, dtype=torch.int8, device="cuda"), torch.empty(6, C // 32, dtype=torch.uint8, device="cuda")
    bm.bimask_ckpt_pack(X, 6, C, q, s)
    q0, s0 = LO.pack(x)
    assert np.array_equal(s.cpu().numpy(), s0)
    assert list(s0[:, 0]) == [255, 1, 248, 1, 255, 248] and list(s0[:, 1]) == [1, 255, 1, 248, 1, 1]
    out = torch.empty(6, C, dtype=torch.bfloat16, device="cuda")
    bm.bimask_ckpt_unpack(q, s, 0, 6, C, out)
    v = out.double().cpu().numpy()
    bad = np.repeat(s0 == 255, 32, axis=1)
    assert np.array_equal(np.isnan(v), bad) and not np.isinf(v).any()
    assert np.array_equal(q.cpu().numpy()[~bad], q0[~bad])
    assert (np.abs(v - x)[~bad] <= TOP / 127.0 / 2).all()    # p / 2 at p = 2^121


def test_pack_at_the_smallest_values():
    """Below 127 * 2^-126 the step stays 2^-126: the error is at most half of it, and no bound relative to the block holds."""
    C = 32
    x = np.outer(np.exp2(np.arange(-133.0, -117.0)), np.linspace(-1.0, 1.0, C))
    X = torch.from_numpy(x).float().to(torch.bfloat16).cuda()
    x = X.double().cpu().numpy()
    q, s = torch.empty(x.shape, dtype=torch.int8, device="cuda"), torch.empty(len(x), 1, dtype=torch.uint8, device="cuda")
    bm.bimask_ckpt_pack(X, len(x), C, q, s)
    q0, s0 = LO.pack(x)
    assert np.array_equal(q.cpu().numpy(), q0) and np.array_equal(s.cpu().numpy(), s0)
    out = torch.empty(len(x), C, dtype=torch.bfloat16, device="cuda")
    bm.bimask_ckpt_unpack(q, s, 0, len(x), C, out)
    p = np.exp2(s0.astype(np.float64) - 127.0)
    assert (np.abs(out.double().cpu().numpy() - x) <= p / 2).all()


# few tokens; pairs; one row tile; two row tiles per CTA; dense operand on pairs and on one row tile
@pytest.mark.parametrize("T,I,J,dense", [(4, 160, 64, False), (200, 288, 64, False), (200, 96, 64, False), (1040, 2080, 4096, False),
                                         (200, 288, 64, True), (200, 96, 64, True), (4, 160, 64, True)])
def test_forward_checkpoint_at_the_largest_values(T, I, J, dense):
    """The product is zero and the bias is the pre-activation, in fp32: one block per case of interest."""
    W = torch.ones(I, J, device="cuda")
    b = bm.alloc_layer_buffers(1, I, J, 1, dense=dense)
    N, M = (4, 8) if dense else (2, 4)
    bm.bimask_fwd_mask(W, I, J, N, M, b["maskbits_f"], b["vals_f"], None if dense else b["meta_f"], None if dense else b["hw_meta_f"])
    bias = np.zeros(I, np.float32)
    bias[3], bias[32], bias[64] = TOP, np.nextafter(np.float32(TOP), np.float32(np.inf)), -MAX
    want_s = [248, 255, 255]
    if I > 128:
        bias[96], bias[128] = 3.4e38, -TOP                   # finite in fp32, infinite in bf16
        want_s += [255, 248]
    X = torch.zeros(T, J, dtype=torch.bfloat16, device="cuda")
    Y = torch.empty(T, I, dtype=torch.bfloat16, device="cuda")
    q, s = torch.empty(T, I, dtype=torch.int8, device="cuda"), torch.empty(T, I // 32, dtype=torch.uint8, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    bm.bimask_linear_fwd(X, b["vals_f"], None if dense else b["hw_meta_f"], torch.from_numpy(bias).cuda(), bm.ACT_NONE, None, T, I, J, Y, q, s, st)
    out = torch.empty(T, I, dtype=torch.bfloat16, device="cuda")
    bm.bimask_ckpt_unpack(q, s, 0, T, I, out)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    s = s.cpu().numpy()
    assert (s[:, :len(want_s)] == want_s).all() and (s[:, len(want_s):] == 1).all()
    v = out.double().cpu().numpy()
    bad = np.repeat(s == 255, 32, axis=1)
    assert np.array_equal(np.isnan(v), bad) and not np.isinf(v).any()
    assert (v[:, 3] == TOP).all() and (I <= 128 or (v[:, 128] == -TOP).all())
