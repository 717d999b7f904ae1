"""The linear-layer operators on the GPU against their plain 64-bit statements.

Tolerances.  A bf16 result must be the rounding of a number that the fp32 evaluation may have given: between the
roundings of y - d and y + d.  For d: the tensor core adds K products in fp32 without rounding to nearest: an absolute error of at most (K / 16 + 32) 2^-23 sum|x w| is allowed for a
sum (one unit in the last place of the running sum per MMA of 16, which is at most 2^-23 sum|x w|).  Activations and
slopes are evaluated to about 1e-6 relative to 1 + |z|; 4e-6 is allowed.  No activation has a slope above 1.13.
Where all sums are exact (small integers) results must be equal bit for bit."""
import numpy as np
import pytest
import torch

import paper_2302_06058_b200 as bm
from oracle import linear_oracle as LO
from paper_2302_06058_b200 import inputs

pytestmark = pytest.mark.gpu


def rounds_from(got, want, d):
    """Element-wise: got (CUDA bf16) lies between the bf16 roundings of want - d and want + d."""
    g = got.double().cpu().numpy()
    return (bf(want - d)[1] <= g) & (g <= bf(want + d)[1])


def cuda(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def bf(a):
    """fp64 array rounded to bf16, as a CUDA tensor and as fp64 again."""
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float64)).float().to(torch.bfloat16)
    return t.cuda(), t.double().numpy()


def operand(W, N, M):
    """(vals, hw_meta, masked bf16 weights as fp64) through the library's mask call, the mask bits read back."""
    I, J = W.shape
    dense = N > 2
    b = bm.alloc_layer_buffers(1, I, J, 1, dense=dense)
    Wd = cuda(W, torch.float32)
    bm.bimask_fwd_mask(Wd, I, J, N, M, b["maskbits_f"], b["vals_f"], None if dense else b["meta_f"], None if dense else b["hw_meta_f"])
    torch.cuda.synchronize()
    bits = np.unpackbits(b["maskbits_f"].cpu().numpy().view(np.uint8), axis=1, bitorder="little")[:, :J]
    Wm = Wd.to(torch.bfloat16).double().cpu().numpy() * bits
    return b["vals_f"], None if dense else b["hw_meta_f"], Wm


def run_linear(vals, hw, X, bias, act, R, T, I, J, ckpt, Y=None, stream=None):
    Y = torch.full((T, I), 7.0, dtype=torch.bfloat16, device="cuda") if Y is None else Y
    q = torch.full((T, I), 99, dtype=torch.int8, device="cuda") if ckpt else None
    s = torch.full((T, I // 32), 77, dtype=torch.uint8, device="cuda") if ckpt else None
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    bm.bimask_linear_fwd(X, vals, hw, bias, act, R, T, I, J, Y, q, s, st, stream)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    return Y, q, s


# tokens x rows x reduction, pattern: one token, a few, one past each tile width, one and several row tiles, reductions
# of one and several tiles and of a part of one, the kernel for long reductions (2048 rows, k >= 4096, 1024 tokens)
SHAPES = [(1, 32, 32, 2, 4), (1, 256, 512, 2, 4), (3, 96, 160, 1, 4), (7, 1152, 384, 2, 4), (31, 384, 1536, 2, 4), (32, 128, 4608, 2, 4),
          (33, 160, 2080, 2, 4), (64, 64, 576, 2, 8), (65, 512, 1024, 1, 16), (127, 416, 96, 2, 4), (128, 1536, 384, 2, 4),
          (129, 128, 384, 2, 4), (300, 96, 288, 2, 4), (257, 288, 416, 2, 4), (1001, 1152, 384, 2, 4), (2048, 384, 384, 1, 4),
          (1056, 2080, 4128, 2, 4), (1024, 2560, 4096, 2, 4),
          (1, 64, 64, 4, 8), (5, 416, 160, 4, 8), (40, 96, 4128, 4, 8), (130, 64, 96, 4, 8), (517, 384, 160, 4, 8), (200, 160, 96, 4, 16)]


@pytest.mark.parametrize("T,I,J,N,M", SHAPES)
def test_forward_exact_on_small_integers(T, I, J, N, M):
    """Sums, bias and residual are small multiples of 1/2: Y (ReLU), the bytes and the scales must be equal."""
    rng = np.random.default_rng(T + I + J)
    W = rng.integers(-2, 3, (I, J)).astype(np.float64) + 0.0
    vals, hw, Wm = operand(W, N, M)
    X, x = bf(rng.integers(-2, 3, (T, J)))
    bias = rng.integers(-9, 10, I) * 0.5
    R, r = bf(rng.integers(-4, 5, (T, I)) * 0.5)
    z = x @ Wm.T + bias
    Y, q, s = run_linear(vals, hw, X, cuda(bias, torch.float32), bm.ACT_RELU, R, T, I, J, True)
    want = torch.from_numpy(np.maximum(z, 0.0) + r).float().to(torch.bfloat16)
    assert torch.equal(Y.cpu(), want)
    q0, s0 = LO.pack(z) if T * I <= 60000 else pack_fast(z)
    assert np.array_equal(s.cpu().numpy(), s0)
    assert np.array_equal(q.cpu().numpy(), q0)


@pytest.mark.parametrize("T,I,J,N,M", [(150, 288, 8224, 2, 4), (129, 1056, 16384, 2, 4), (300, 160, 4128, 4, 8), (260, 416, 8192, 1, 4)])
def test_forward_exact_where_many_tokens_split_the_reduction(T, I, J, N, M):
    """More than one 128-token tile on the kernel for few tokens (long reductions with few output tiles), ragged at both ends."""
    test_forward_exact_on_small_integers(T, I, J, N, M)


def pack_fast(z):
    b = z.reshape(z.shape[0], -1, 32)
    m = np.abs(b).max(-1)
    e = np.full(m.shape, -126)
    for k in range(-126, 121):
        e = np.where(m > 127.0 * 2.0 ** k, k + 1, e)
    q = np.rint(b / np.exp2(e)[..., None]).astype(np.int8)
    return q.reshape(z.shape), (e + 127).astype(np.uint8)


def test_fast_pack_of_this_file_is_the_plain_one():
    z = np.random.default_rng(1).standard_normal((6, 64)) * 50
    a, b = LO.pack(z), pack_fast(z)
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


@pytest.mark.parametrize("act", LO.ACTS)
@pytest.mark.parametrize("T,I,J,N,M", [(1, 288, 1184, 2, 4), (30, 96, 2304, 2, 4), (77, 160, 96, 1, 4), (300, 64, 160, 2, 4),
                                       (350, 416, 384, 2, 4), (1100, 2144, 4096, 2, 4), (20, 160, 512, 4, 8), (190, 288, 160, 4, 8)])
def test_forward_against_64_bits(act, T, I, J, N, M):
    rng = np.random.default_rng(7 * T + act)
    W = inputs.make_weight(I, J, 11 + I).astype(np.float64)
    vals, hw, Wm = operand(W, N, M)
    X, x = bf(rng.standard_normal((T, J)) * 1.5)
    bias = rng.standard_normal(I).astype(np.float32)
    R, r = bf(rng.standard_normal((T, I)))
    for use_b, use_r, use_c in ((True, True, True), (False, False, False), (True, False, True), (False, True, False)):
        y, z = LO.linear(x, Wm, bias if use_b else None, act, r if use_r else None)
        Y, q, s = run_linear(vals, hw, X, cuda(bias) if use_b else None, act, R if use_r else None, T, I, J, use_c)
        acc = (J / 16 + 32) * 2.0 ** -23 * (np.abs(x) @ np.abs(Wm).T + np.abs(bias))
        assert rounds_from(Y, y, 1.2 * acc + 4e-6 * (1.0 + np.abs(z))).all()
        if use_c:
            v = LO.unpack(q.cpu().numpy(), s.cpu().numpy())
            p = np.repeat(np.exp2(s.cpu().numpy().astype(np.float64) - 127.0), 32, axis=1)
            assert (np.abs(v - z) <= p / 2 + acc).all()
            top = np.repeat(np.abs(z.reshape(T, -1, 32)).max(-1), 32, axis=1)
            worst = np.repeat(acc.reshape(T, -1, 32).max(-1), 32, axis=1)
            assert (top - worst <= 127.0 * p).all() and (top + worst > 127.0 * p / 2).all()


@pytest.mark.parametrize("T,I,J", [(9, 96, 160), (200, 64, 96), (300, 288, 160), (1040, 2080, 4096)])
def test_forward_residual_may_be_the_result(T, I, J):
    rng = np.random.default_rng(T)
    vals, hw, _ = operand(rng.standard_normal((I, J)), 2, 4)
    X, _ = bf(rng.standard_normal((T, J)))
    R, _ = bf(rng.standard_normal((T, I)))
    a, _, _ = run_linear(vals, hw, X, None, bm.ACT_SILU, R, T, I, J, False)
    both = R.clone()
    b, _, _ = run_linear(vals, hw, X, None, bm.ACT_SILU, both, T, I, J, False, Y=both)
    assert torch.equal(a, b)


def test_forward_plain_layer_is_the_bare_product():
    """Without bias, activation and residual the result is bimask_spmm_fwd's, bit for bit, where the kernels agree."""
    for T, I, J in ((300, 384, 384), (1040, 2080, 4096), (300, 64, 96)):
        vals, hw, _ = operand(np.random.default_rng(I).standard_normal((I, J)), 2, 4)
        X, _ = bf(np.random.default_rng(J).standard_normal((T, J)))
        Y0 = torch.empty(T, I, dtype=torch.bfloat16, device="cuda")
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        bm.bimask_spmm_fwd(X, vals, hw, T, I, J, Y0, st)
        Y, _, _ = run_linear(vals, hw, X, None, 0, None, T, I, J, False)
        assert torch.equal(Y, Y0)


@pytest.mark.parametrize("T,I,J,N,M", [(2, 64, 96, 2, 4), (50, 96, 4128, 2, 4), (140, 64, 160, 2, 4), (333, 160, 96, 2, 4),
                                       (1030, 2080, 4096, 2, 4), (333, 160, 96, 4, 8), (33, 96, 160, 4, 8)])
def test_forward_writes_nothing_outside_its_results(T, I, J, N, M):
    vals, hw, _ = operand(np.random.default_rng(2).standard_normal((I, J)), N, M)
    X, _ = bf(np.random.default_rng(3).standard_normal((T, J)))
    R, _ = bf(np.random.default_rng(4).standard_normal((T, I)))
    pad = 4096

    def guarded(n, dtype, fill):
        t = torch.full((n + 2 * pad,), fill, dtype=dtype, device="cuda")
        return t, t[pad:pad + n]

    yb, Y = guarded(T * I, torch.bfloat16, 3.0)
    qb, q = guarded(T * I, torch.int8, 55)
    sb, s = guarded(T * I // 32, torch.uint8, 66)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    bm.bimask_linear_fwd(X, vals, hw, None, bm.ACT_GELU, R, T, I, J, Y, q, s, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    for b, n, fill in ((yb, T * I, 3.0), (qb, T * I, 55), (sb, T * I // 32, 66)):
        assert bool((b[:pad] == fill).all()) and bool((b[pad + n:] == fill).all())


@pytest.mark.parametrize("T,I,J", [(6, 96, 160), (140, 64, 96), (300, 288, 160), (1030, 2080, 4096)])
def test_forward_non_finite_and_empty_rows(T, I, J):
    """A NaN or an infinity in one token stays in that token and in the rows of W that keep its column; a token of zeros
    and a zero row of W leave the bias alone; the checkpoint marks exactly the blocks that are not finite."""
    rng = np.random.default_rng(T)
    W = rng.standard_normal((I, J))
    W[5] = 0.0
    vals, hw, Wm = operand(W, 2, 4)
    xs = rng.standard_normal((T, J))
    xs[1, 3], xs[2, 4], xs[3] = np.nan, np.inf, 0.0
    X, x = bf(xs)
    bias = rng.standard_normal(I).astype(np.float32)
    Y, q, s = run_linear(vals, hw, X, cuda(bias), bm.ACT_RELU, None, T, I, J, True)
    Y, s = Y.double().cpu().numpy(), s.cpu().numpy()
    fine = np.ones(T, bool)
    fine[1:3] = False
    assert np.isfinite(Y[fine]).all() and (s[fine] != 255).all()
    kept = Wm != 0                                            # no kept weight is zero outside row 5, which keeps columns 0 and 1 mod 4
    assert np.array_equal(np.isnan(Y[1]), kept[:, 3])
    assert np.array_equal(np.isinf(Y[2]), Wm[:, 4] > 0) and np.array_equal(np.isnan(Y[2]), np.arange(I) == 5)      # infinity times a kept zero
    for t, col in ((1, 3), (2, 4)):
        assert np.array_equal(s[t] == 255, (kept[:, col] | ((np.arange(I) == 5) & (col % 4 < 2))).reshape(-1, 32).any(-1))
    want = torch.from_numpy(np.maximum(bias, 0)).to(torch.bfloat16).double().numpy()
    assert np.array_equal(Y[3], want)
    assert np.array_equal(Y[fine, 5], np.full(fine.sum(), want[5]))     # the zero row
    v = LO.unpack(q.cpu().numpy(), s)
    assert np.array_equal(np.isnan(v[1]), np.repeat(s[1] == 255, 32)) and np.isfinite(v[fine]).all()


def test_forward_large_bias_overflows_like_bf16():
    T, I, J = 4, 64, 64
    vals, hw, _ = operand(np.random.default_rng(0).standard_normal((I, J)), 2, 4)
    X, _ = bf(np.zeros((T, J)))
    bias = np.zeros(I, np.float32)
    bias[0], bias[33] = 3.3e38, 3.4e38                       # below and above the largest finite bf16
    Y, q, s = run_linear(vals, hw, X, cuda(bias), 0, None, T, I, J, True)
    assert bool(torch.isfinite(Y[:, 0]).all()) and bool(torch.isinf(Y[:, 33]).all())
    assert (s[:, 0] == 248).all() and (s[:, 1] == 255).all()


@pytest.mark.parametrize("T,C", [(1, 32), (1, 16384), (2, 64), (3, 96), (5, 4128), (31, 384), (64, 2080), (100, 1536), (1000, 32), (777, 160),
                                 (4099, 64)])
def test_checkpoint_bit_exact(T, C):
    rng = np.random.default_rng(T + C)
    x = rng.standard_normal((T, C)) * np.exp2(rng.integers(-30, 30, (T, 1)))
    if T > 2:
        x[0], x[1, :31], x[1, 31] = 0.0, 127.0, -0.0
        x[2, 0:32] = 2.0 ** -133                              # subnormal in bf16
        x[2, C - 1] = 3.0e38
    X, x = bf(x)
    if T > 4:
        X[3, 1], X[4, C - 1] = float("nan"), float("-inf")
        x[3, 1], x[4, C - 1] = np.nan, -np.inf
    q = torch.empty(T, C, dtype=torch.int8, device="cuda")
    s = torch.empty(T, C // 32, dtype=torch.uint8, device="cuda")
    bm.bimask_ckpt_pack(X, T, C, q, s)
    out = torch.empty(T, C, dtype=torch.bfloat16, device="cuda")
    bm.bimask_ckpt_unpack(q, s, 0, T, C, out)
    q, s, out = q.cpu().numpy(), s.cpu().numpy(), out.double().cpu().numpy()
    if T * C <= 70000:
        q0, s0 = LO.pack(x)
    else:
        q0, s0 = pack_fast(np.nan_to_num(x, nan=0.0, posinf=0.0, neginf=0.0))
        bad = ~np.isfinite(x).reshape(T, -1, 32).all(-1)
        s0[bad] = 255
    assert np.array_equal(s, s0)
    ok = np.repeat(s0 != 255, 32, axis=1)
    assert np.array_equal(q[ok], q0[ok])
    v = LO.unpack(q0, s0)
    assert np.array_equal(np.isnan(out), ~ok) and np.array_equal(out[ok], v[ok])


@pytest.mark.parametrize("act", LO.ACTS)
def test_restore_through_an_activation(act):
    T, C = 37, 224
    rng = np.random.default_rng(act)
    q = rng.integers(-127, 128, (T, C)).astype(np.int8)
    s = rng.integers(112, 126, (T, C // 32)).astype(np.uint8)
    s[0, 0], s[1, 1], s[2, 2] = 1, 255, 200
    z = LO.unpack(q, s)
    out = torch.empty(T, C, dtype=torch.bfloat16, device="cuda")
    bm.bimask_ckpt_unpack(cuda(q), cuda(s), act, T, C, out)
    got = out.double().cpu().numpy()
    with np.errstate(all="ignore"):
        want = LO.act(z, act)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    ok = ~np.isnan(want)
    assert rounds_from(out, np.nan_to_num(want), np.nan_to_num(4e-6 * np.minimum(1.0 + np.abs(z), 10.0)))[ok].all()


@pytest.mark.parametrize("act", LO.ACTS)
@pytest.mark.parametrize("T,C", [(1, 32), (1, 2080), (2, 96), (33, 384), (130, 1536), (515, 64), (70, 4128), (1024, 160)])
def test_gradient_of_the_epilogue(act, T, C):
    rng = np.random.default_rng(3 * T + C + act)
    dY, dy = bf(rng.standard_normal((T, C)))
    q, s = pack_fast(rng.standard_normal((T, C)) * 2.0)
    z = LO.unpack(q, s)
    dz, db = LO.act_bwd(dy, z, act)
    ws = torch.empty(bm.bimask_linear_workspace_bytes(T, C, 32), dtype=torch.uint8, device="cuda")
    dZ = torch.full((T, C), 9.0, dtype=torch.bfloat16, device="cuda")
    dB = torch.full((C,), 9.0, device="cuda")
    zq, zs = (None, None) if act == 0 else (cuda(q), cuda(s))
    bm.bimask_act_bwd(dY, zq, zs, act, T, C, dZ, dB, ws, ws.numel())
    gb = dB.double().cpu().numpy()
    assert rounds_from(dZ, dz, 4e-6 * np.abs(dy)).all()
    assert (np.abs(gb - db) <= (T + 64) * 2.0 ** -24 * np.abs(dz).sum(0) + 4e-6 * np.abs(dy).sum(0)).all()
    h = 1e-5                                                  # and against differences of the activation
    with np.errstate(all="ignore"):
        diff = (LO.act(z + h, act) - LO.act(z - h, act)) / (2 * h)
    smooth = np.abs(z) > 2 * h if act == LO.RELU else np.ones_like(z, bool)
    assert rounds_from(dZ, np.where(smooth, dy * diff, dz), 5e-6 * np.abs(dy)).all()
    # each result alone, and the gradient in place
    only = torch.empty(C, device="cuda")
    bm.bimask_act_bwd(dY, zq, zs, act, T, C, None, only, ws, ws.numel())
    assert torch.equal(only, dB)
    same = dY.clone()
    bm.bimask_act_bwd(same, zq, zs, act, T, C, same, None, None, 0)
    assert torch.equal(same, dZ)


def test_gradient_of_the_epilogue_bad_blocks_and_extremes():
    """A block that was not finite gives NaN in its own channels only; far tails give slopes 0 and 1."""
    T, C = 6, 96
    q = np.full((T, C), 127, np.int8)
    q[3] = -127
    s = np.full((T, C // 32), 130, np.uint8)                  # z = +-1016
    s[1, 1] = 255
    s[4], s[5] = 240, 240
    q[5] = -127
    dY = torch.ones(T, C, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(bm.bimask_linear_workspace_bytes(T, C, 32), dtype=torch.uint8, device="cuda")
    for act in (bm.ACT_RELU, bm.ACT_GELU, bm.ACT_GELU_TANH, bm.ACT_SILU):
        dZ, db = torch.empty_like(dY), torch.empty(C, device="cuda")
        bm.bimask_act_bwd(dY, cuda(q), cuda(s), act, T, C, dZ, db, ws, ws.numel())
        d = dZ.float().cpu()
        nan = torch.isnan(d)
        assert bool(nan[1, 32:64].all()) and int(nan.sum()) == 32
        assert bool((d[[0, 2, 4]] == 1).all()) and bool((d[[3, 5]] == 0).all())
        assert bool(torch.isnan(db[32:64]).all()) and bool(torch.isfinite(db[:32]).all())


@pytest.mark.parametrize("T,I,J", [(1, 32, 32), (3, 96, 64), (64, 128, 256), (65, 160, 288), (500, 64, 576), (1000, 384, 384), (4096, 96, 96),
                                   (777, 1152, 384), (9000, 288, 544), (16500, 512, 4608)])
def test_weight_gradient_from_a_checkpoint(T, I, J):
    rng = np.random.default_rng(T + J)
    dY, dy = bf(rng.standard_normal((T, I)))
    q, s = pack_fast(rng.standard_normal((T, J)) * 3.0)
    ws = torch.empty(bm.bimask_linear_workspace_bytes(T, I, J), dtype=torch.uint8, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    dW = torch.full((I, J), 5.0, device="cuda")
    bm.bimask_wgrad_ckpt(dY, cuda(q), cuda(s), T, I, J, dW, ws, ws.numel(), st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    x = LO.unpack(q, s)
    xd, yd = cuda(x), cuda(dy)
    want, size = yd.t() @ xd, yd.abs().t() @ xd.abs()
    chain = min(T, 8192)
    assert bool(((dW.double() - want).abs() <= (chain / 16 + 64) * 2.0 ** -23 * size).all())
    assert float((dW.double() - want).norm() / want.norm()) < 2e-5


def test_weight_gradient_from_a_checkpoint_exact_and_strayless():
    """Integer values and gradients: equal bit for bit, nothing written outside, a NaN block in its own columns only."""
    T, I, J = 333, 160, 224
    rng = np.random.default_rng(8)
    dY, dy = bf(rng.integers(-3, 4, (T, I)))
    q = rng.integers(-127, 128, (T, J)).astype(np.int8)
    s = np.full((T, J // 32), 127, np.uint8)
    n = bm.bimask_linear_workspace_bytes(T, I, J)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    buf = torch.full((I * J + 8192,), 3.0, device="cuda")
    dW = buf[4096:4096 + I * J]
    bm.bimask_wgrad_ckpt(dY, cuda(q), cuda(s), T, I, J, dW, ws, n, st)
    assert np.array_equal(dW.view(I, J).double().cpu().numpy(), dy.T @ q.astype(np.float64))
    assert bool((buf[:4096] == 3).all()) and bool((buf[4096 + I * J:] == 3).all())
    s[7, 2] = 255
    bm.bimask_wgrad_ckpt(dY, cuda(q), cuda(s), T, I, J, dW, ws, n, st)
    nan = torch.isnan(dW.view(I, J)).cpu()
    assert bool(nan[:, 64:96].all()) and int(nan.sum()) == 32 * I


def test_other_streams_and_graphs():
    """Every call on a stream of its own, captured and replayed on changed inputs."""
    T, I, J = 200, 288, 384
    rng = np.random.default_rng(1)
    vals, hw, _ = operand(rng.standard_normal((I, J)), 2, 4)
    X, _ = bf(rng.standard_normal((T, J)))
    X2, _ = bf(rng.standard_normal((T, J)))
    dY, _ = bf(rng.standard_normal((T, I)))
    bias = torch.randn(I, device="cuda")
    n = bm.bimask_linear_workspace_bytes(T, I, J)

    def buffers():
        e = lambda *s, dtype=torch.bfloat16: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
        return {"Y": e(T, I), "zq": e(T, I, dtype=torch.int8), "zs": e(T, I // 32, dtype=torch.uint8), "xq": e(T, J, dtype=torch.int8),
                "xs": e(T, J // 32, dtype=torch.uint8), "dZ": e(T, I), "db": e(I, dtype=torch.float32), "dW": e(I, J, dtype=torch.float32),
                "H": e(T, I), "ws": e(n, dtype=torch.uint8), "st": torch.zeros(1, dtype=torch.int32, device="cuda")}

    def step(x, b, stream=None):
        bm.bimask_ckpt_pack(x, T, J, b["xq"], b["xs"], stream)
        bm.bimask_linear_fwd(x, vals, hw, bias, bm.ACT_GELU, None, T, I, J, b["Y"], b["zq"], b["zs"], b["st"], stream)
        bm.bimask_ckpt_unpack(b["zq"], b["zs"], bm.ACT_GELU, T, I, b["H"], stream)
        bm.bimask_act_bwd(dY, b["zq"], b["zs"], bm.ACT_GELU, T, I, b["dZ"], b["db"], b["ws"], n, stream)
        bm.bimask_wgrad_ckpt(b["dZ"], b["xq"], b["xs"], T, I, J, b["dW"], b["ws"], n, b["st"], stream)

    keys = ("Y", "zq", "zs", "dZ", "db", "dW", "H")
    one, two = buffers(), buffers()
    step(X, one)
    step(X2, two)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    b = buffers()
    side.wait_stream(torch.cuda.current_stream())
    step(X, b, side)
    side.synchronize()
    for k in keys:
        assert torch.equal(b[k], one[k]), k
    x, b = X.clone(), buffers()
    with torch.cuda.stream(side):
        step(x, b)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        step(x, b)
    for src, want in ((X2, two), (X, one)):
        x.copy_(src)
        g.replay()
        torch.cuda.synchronize()
        for k in keys:
            assert torch.equal(b[k], want[k]), k
    assert int(b["st"].item()) == 0


def test_repeated_runs_are_identical():
    T, I, J = 1500, 96, 4128
    rng = np.random.default_rng(6)
    dY, _ = bf(rng.standard_normal((T, I)))
    q, s = pack_fast(rng.standard_normal((T, I)))
    ws = torch.empty(bm.bimask_linear_workspace_bytes(T, I, J), dtype=torch.uint8, device="cuda")
    out = []
    for _ in range(3):
        dZ, db = torch.empty(T, I, dtype=torch.bfloat16, device="cuda"), torch.empty(I, device="cuda")
        bm.bimask_act_bwd(dY, cuda(q), cuda(s), bm.ACT_SILU, T, I, dZ, db, ws, ws.numel())
        out.append((dZ, db))
    assert all(torch.equal(a, b) for o in out[1:] for a, b in zip(out[0], o))


def test_offsets_past_32_bits():
    """More than 2^31 elements: the last token's results must be those of the same token alone."""
    T, C = 262145, 8192 + 32
    n = T * C
    assert n > 1 << 31
    x = torch.zeros(T, C, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(4)
    x[-3:] = torch.randn(3, C, generator=g, device="cuda").to(torch.bfloat16)
    q = torch.empty(T, C, dtype=torch.int8, device="cuda")
    s = torch.empty(T, C // 32, dtype=torch.uint8, device="cuda")
    bm.bimask_ckpt_pack(x, T, C, q, s)
    q0 = torch.empty(3, C, dtype=torch.int8, device="cuda")
    s0 = torch.empty(3, C // 32, dtype=torch.uint8, device="cuda")
    bm.bimask_ckpt_pack(x[-3:].contiguous(), 3, C, q0, s0)
    assert torch.equal(q[-3:], q0) and torch.equal(s[-3:], s0) and not bool(q[:-3].any())
    ws = torch.empty(bm.bimask_linear_workspace_bytes(T, C, 32), dtype=torch.uint8, device="cuda")
    db = torch.empty(C, device="cuda")
    bm.bimask_act_bwd(x, q, s, bm.ACT_GELU, T, C, x, db, ws, ws.numel())
    dz = torch.empty(3, C, dtype=torch.bfloat16, device="cuda")
    db0 = torch.empty(C, device="cuda")
    g.manual_seed(4)
    d0 = torch.randn(3, C, generator=g, device="cuda").to(torch.bfloat16)
    bm.bimask_act_bwd(d0, q0, s0, bm.ACT_GELU, 3, C, dz, db0, ws, ws.numel())
    assert torch.equal(x[-3:], dz) and torch.allclose(db, db0, atol=1e-6)
    bm.bimask_ckpt_unpack(q, s, 0, T, C, x)
    bm.bimask_ckpt_unpack(q0, s0, 0, 3, C, dz)
    assert torch.equal(x[-3:], dz)


def test_forward_offsets_past_32_bits():
    """More than 2^31 results: the last tokens' results and checkpoint must be those of the same tokens alone."""
    T, I, J, last = 131201, 16416, 64, 150
    assert T * I > 1 << 31
    vals, hw, _ = operand(np.random.default_rng(1).standard_normal((I, J)), 2, 4)
    g = torch.Generator(device="cuda").manual_seed(2)
    X = torch.randn(T, J, generator=g, device="cuda").to(torch.bfloat16)
    bias = torch.randn(I, generator=g, device="cuda")
    Y, q, s = run_linear(vals, hw, X, bias, bm.ACT_GELU, None, T, I, J, True)
    Y0, q0, s0 = run_linear(vals, hw, X[-last:].contiguous(), bias, bm.ACT_GELU, None, last, I, J, True)
    assert torch.equal(Y[-last:], Y0) and torch.equal(q[-last:], q0) and torch.equal(s[-last:], s0)
    R = Y
    Y2, _, _ = run_linear(vals, hw, X, None, bm.ACT_NONE, R, T, I, J, False, Y=R)
    Y3, _, _ = run_linear(vals, hw, X[-last:].contiguous(), None, bm.ACT_NONE, Y0.clone(), last, I, J, False)
    assert torch.equal(Y2[-last:], Y3)
