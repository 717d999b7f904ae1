"""Dropout on the GPU: masks bit for bit against the published generator, values against one rounding."""
import numpy as np
import pytest
import torch

import paper_2302_06058_b200 as bm
from oracle import linear_oracle as LO
from oracle import residual_oracle as RO

pytestmark = pytest.mark.gpu
SEED, NUMBER = 0x0123456789ABCDEF, 0xFEDCBA9876543210
DTYPES = {"bf16": (torch.bfloat16, bm.TYPE_BF16), "f32": (torch.float32, bm.TYPE_F32)}


def expected(x, p, seed=SEED, number=NUMBER, first_row=0):
    """x (CUDA, contiguous rows) dropped: the product in fp32, rounded to x's type; a CPU tensor."""
    T, C = x.shape
    thr = RO.threshold(p)
    if thr == 0:
        return x.cpu()
    y = (x.float().cpu() * float(np.float32(65536.0 / (65536 - thr)))).to(x.dtype)
    return torch.where(torch.from_numpy(RO.keep(T, C, p, seed, number, first_row)), y, torch.zeros((), dtype=x.dtype))


def same(a, b):
    """Equal bit for bit."""
    i = torch.int16 if a.dtype == torch.bfloat16 else torch.int32
    return torch.equal(a.cpu().contiguous().view(i), b.cpu().contiguous().view(i))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.99999])
@pytest.mark.parametrize("T,C", [(1, 32), (3, 96), (1001, 1152), (257, 4096), (5, 16384)])
def test_values_and_masks(T, C, p, dtype):
    dt, code = DTYPES[dtype]
    x = torch.randn(T, C, generator=torch.Generator().manual_seed(T + C)).to(dt).cuda()
    y = torch.full_like(x, 7.0)
    d = bm.make_dropout(p, SEED, NUMBER)
    bm.bimask_dropout(x, code, T, C, d, y)
    assert same(y, expected(x, p))
    bm.bimask_dropout(x, code, T, C, d, x)                                  # in place
    assert same(x, y)


@pytest.mark.parametrize("dtype", DTYPES)
def test_dropped_values_are_zero_whatever_they_were(dtype):
    dt, code = DTYPES[dtype]
    x = torch.tensor([float("nan"), float("inf"), -float("inf"), 3.0e38, -0.0, 1.0, -1.0, 1e-40], dtype=torch.float32).repeat(64, 8).to(dt).cuda()
    y = torch.empty_like(x)
    bm.bimask_dropout(x, code, 64, 64, bm.make_dropout(0.5, SEED, NUMBER), y)
    keep = torch.from_numpy(RO.keep(64, 64, 0.5, SEED, NUMBER))
    want = expected(x, 0.5)
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(y).cpu(), nan & keep)
    assert same(torch.where(nan, torch.zeros((), dtype=dt), want), torch.where(nan, torch.zeros((), dtype=dt), y.cpu()))


def test_counter_in_device_memory_and_a_replayed_graph():
    """The counter is read when the kernel runs: every replay of a captured call draws the mask of its own step; two graphs that
    share buffers and counter draw what their stream numbers say."""
    T, C, p = 40, 96, 0.3
    x = torch.randn(T, C, device="cuda").to(torch.bfloat16)
    ys = [torch.empty_like(x) for _ in range(2)]
    counter = torch.zeros(1, dtype=torch.int64, device="cuda")
    drops = [bm.make_dropout(p, SEED, (1 << 32) - 2 + 10 * i, counter) for i in range(2)]
    for d, y in zip(drops, ys):
        bm.bimask_dropout(x, bm.TYPE_BF16, T, C, d, y)
    graphs = []
    for d, y in zip(drops, ys):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            bm.bimask_dropout(x, bm.TYPE_BF16, T, C, d, y)
        graphs.append(g)
    for step in (0, 1, 2, 5):                                              # passes 2^32 in the first graph's number
        counter.fill_(step)
        for i in (1, 0):
            graphs[i].replay()
        torch.cuda.synchronize()
        for i in (0, 1):
            assert same(ys[i], expected(x, p, number=(1 << 32) - 2 + 10 * i + step))


def test_another_stream_and_nothing_outside_the_result():
    T, C, pad = 77, 160, 4096
    x = torch.randn(T, C, device="cuda").to(torch.bfloat16)
    buf = torch.full((T * C + 2 * pad,), 3.0, dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    bm.bimask_dropout(x, bm.TYPE_BF16, T, C, bm.make_dropout(0.2, SEED, NUMBER), buf[pad:pad + T * C], stream=side)
    side.synchronize()
    assert same(buf[pad:pad + T * C].view(T, C), expected(x, 0.2))
    assert bool((buf[:pad] == 3.0).all()) and bool((buf[pad + T * C:] == 3.0).all())


def test_more_than_2_31_elements():
    C = 16384
    T = (1 << 31) // C + 5
    x = torch.ones(T, C, dtype=torch.bfloat16, device="cuda")
    bm.bimask_dropout(x, bm.TYPE_BF16, T, C, bm.make_dropout(0.25, SEED, NUMBER), x)
    ones = torch.ones(3, C, dtype=torch.bfloat16)
    for row in (0, T // 2, T - 8, T - 3):
        assert same(x[row:row + 3], expected(ones, 0.25, first_row=row))


def bf16_between(got, lo, hi):
    def r(a):
        return torch.from_numpy(np.ascontiguousarray(a)).float().to(torch.bfloat16).double().numpy()
    g = got.double().cpu().numpy()
    return (r(lo) <= g) & (g <= r(hi))


@pytest.mark.parametrize("act", LO.ACTS)
@pytest.mark.parametrize("T,C,p", [(1, 32, 0.5), (33, 160, 0.1), (700, 1536, 0.3), (9, 16384, 0.25)])
def test_hidden_layer_recomputed_and_its_gradient(act, T, C, p):
    """Activations are evaluated to 1e-6 (1 + |z|), slopes to 1e-6 (4e-6 allowed, as for the calls without dropout), times the
    multiplier; bias sums add at most T values in fp32."""
    rng = np.random.default_rng(T + act)
    X = torch.from_numpy(rng.standard_normal((T, C)) * 2).to(torch.bfloat16).cuda()
    q, s = torch.empty(T, C, dtype=torch.int8, device="cuda"), torch.empty(T, C // 32, dtype=torch.uint8, device="cuda")
    bm.bimask_ckpt_pack(X, T, C, q, s)
    z = LO.unpack(q.cpu().numpy(), s.cpu().numpy())
    d = bm.make_dropout(p, SEED, NUMBER)
    m = RO.multiplier(T, C, p, SEED, NUMBER)
    H = torch.full((T, C), 7.0, dtype=torch.bfloat16, device="cuda")
    bm.bimask_ckpt_unpack_dropout(q, s, act, d, T, C, H)
    want, tol = LO.act(z, act) * m, (4e-6 * (1 + np.abs(z)) + 1e-6 * np.abs(z)) * m
    assert bf16_between(H, want - tol, want + tol).all()
    dY = torch.from_numpy(rng.standard_normal((T, C))).to(torch.bfloat16).cuda()
    ws = torch.empty(bm.bimask_linear_workspace_bytes(T, C, 32), dtype=torch.uint8, device="cuda")
    dZ, db = torch.full_like(dY, 7.0), torch.full((C,), 7.0, device="cuda")
    bm.bimask_act_dropout_bwd(dY, q, s, act, d, T, C, dZ, db, ws, ws.numel())
    dy = dY.double().cpu().numpy()
    want, tol = dy * m * LO.slope(z, act), 5e-6 * np.abs(dy) * m
    assert bf16_between(dZ, want - tol, want + tol).all()
    assert (np.abs(db.double().cpu().numpy() - want.sum(0)) <= tol.sum(0) + (T + 8) * 2.0 ** -24 * np.abs(want).sum(0)).all()
    both = dY.clone()
    only = torch.empty_like(db)
    bm.bimask_act_dropout_bwd(both, q, s, act, d, T, C, both, None, None, 0)               # in place, without the bias
    bm.bimask_act_dropout_bwd(dY, q, s, act, d, T, C, None, only, ws, ws.numel())          # the bias alone
    assert same(both, dZ) and torch.equal(only, db)


def test_without_dropout_the_calls_are_the_plain_ones():
    T, C = 50, 96
    X = torch.randn(T, C, device="cuda").to(torch.bfloat16)
    q, s = torch.empty(T, C, dtype=torch.int8, device="cuda"), torch.empty(T, C // 32, dtype=torch.uint8, device="cuda")
    bm.bimask_ckpt_pack(X, T, C, q, s)
    ws = torch.empty(bm.bimask_linear_workspace_bytes(T, C, 32), dtype=torch.uint8, device="cuda")
    a, b = torch.empty_like(X), torch.empty_like(X)
    da, db = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    none = bm.make_dropout(0.0, SEED)
    bm.bimask_ckpt_unpack(q, s, bm.ACT_GELU, T, C, a)
    bm.bimask_ckpt_unpack_dropout(q, s, bm.ACT_GELU, none, T, C, b)
    assert same(a, b)
    bm.bimask_act_bwd(X, q, s, bm.ACT_GELU, T, C, a, da, ws, ws.numel())
    bm.bimask_act_dropout_bwd(X, q, s, bm.ACT_GELU, none, T, C, b, db, ws, ws.numel())
    assert same(a, b) and torch.equal(da, db)
