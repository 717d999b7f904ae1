"""CPU checks of the linear-layer operators: the plain 64-bit statements against closed forms, differences and torch's
own functions, and the refusals of the library's entry points (no GPU is touched)."""
import math

import numpy as np
import pytest
import torch

from oracle import linear_oracle as LO


@pytest.fixture(scope="module")
def bm():
    from paper_2302_06058_b200 import build
    build.build()
    import paper_2302_06058_b200 as m
    m.lib()
    return m


TORCH = {LO.NONE: lambda z: z, LO.RELU: torch.relu, LO.GELU: torch.nn.functional.gelu,
         LO.GELU_TANH: lambda z: torch.nn.functional.gelu(z, approximate="tanh"), LO.SILU: torch.nn.functional.silu}


@pytest.mark.parametrize("kind", LO.ACTS)
def test_activations_and_slopes_against_autograd_and_differences(kind):
    z = np.concatenate([np.linspace(-9, 9, 181) + 0.013, [-30.0, 30.0, 1e-9]])
    zt = torch.from_numpy(z.copy()).requires_grad_()
    y = TORCH[kind](zt)
    y.sum().backward()
    assert np.allclose(LO.act(z, kind), y.detach().numpy(), rtol=1e-12, atol=1e-14)
    assert np.allclose(LO.slope(z, kind), zt.grad.numpy(), rtol=1e-10, atol=1e-12)
    h = 1e-5
    d = (LO.act(z + h, kind) - LO.act(z - h, kind)) / (2 * h)
    keep = np.abs(z) > 2 * h if kind == LO.RELU else np.ones_like(z, bool)
    assert np.allclose(LO.slope(z, kind)[keep], d[keep], atol=1e-8)


def test_checkpoint_by_hand():
    """One block whose largest value sits just below, at, and above 127 steps of a power of two."""
    x = np.zeros((1, 32))
    x[0, :4] = [127.0, -126.5, 0.5, 1.5]
    q, s = LO.pack(x)
    assert s[0, 0] == 127 and list(q[0, :4]) == [127, -126, 0, 2]          # step 1; ties to even
    x[0, 0] = 127.5
    q, s = LO.pack(x)
    assert s[0, 0] == 128 and q[0, 0] == 64 and q[0, 1] == -63             # step 2: 63.75 -> 64, -63.25 -> -63
    x[0, 0] = 254.0
    q, s = LO.pack(x)
    assert s[0, 0] == 128 and q[0, 0] == 127
    q, s = LO.pack(np.zeros((2, 64)))
    assert (s == 1).all() and (q == 0).all()
    x[0, 0] = np.inf
    q, s = LO.pack(x)
    assert s[0, 0] == 255 and np.isnan(LO.unpack(q, s)).all()


def test_checkpoint_values_are_exact_in_bf16_and_near():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((40, 96)) * np.exp2(rng.integers(-40, 40, (40, 1)))
    q, s = LO.pack(x)
    v = LO.unpack(q, s)
    assert np.array_equal(torch.from_numpy(v).to(torch.bfloat16).double().numpy(), v)
    p = np.repeat(np.exp2(s.astype(np.float64) - 127), 32, axis=1)
    assert (np.abs(v - x) <= p / 2).all()
    top = np.repeat(np.abs(x.reshape(40, 3, 32)).max(-1), 32, axis=1)
    assert (p <= 2 * top / 127).all() and (top <= 127 * p).all()
    assert np.array_equal(LO.unpack(*LO.pack(v)), v)                       # a checkpoint of the values is the values


def test_bias_gradient_by_differences():
    """The loss sum(dY act(z + b)): its derivative by b is the column sum of dY act'(z)."""
    rng = np.random.default_rng(5)
    z, dY, h = rng.standard_normal((9, 32)), rng.standard_normal((9, 32)), 1e-6
    for kind in (LO.GELU, LO.GELU_TANH, LO.SILU):
        _, db = LO.act_bwd(dY, z, kind)
        d = ((dY * LO.act(z + h, kind)).sum(0) - (dY * LO.act(z - h, kind)).sum(0)) / (2 * h)
        assert np.allclose(db, d, atol=1e-7)


def test_workspace_query(bm):
    q = bm.bimask_linear_workspace_bytes
    assert q(0, 64, 64) == 0 and q(4, 48, 64) == 0 and q(4, 64, 48) == 0 and q(-1, 64, 64) == 0
    assert q(1, 32, 32) >= 64
    assert q(8192, 16384, 4096) >= 2 * 8192 * 4096          # many output tiles: the checkpoint is unpacked into it
    assert q(12608, 384, 1536) >= 2 * 4 * 384 * 1536         # few: partial sums of several pieces of the tokens


def test_refusals_name_the_cause(bm):
    """Every bad argument is refused on the host, before any launch."""
    L = bm.lib()
    inval = bm.binding.BIMASK_EINVAL
    n0 = bm.bimask_launch_count()
    a, odd = 256, 264                                       # addresses that are never dereferenced: aligned, misaligned

    def lin(X=a, vals=a, hw=a, bias=None, act=0, R=None, T=4, I=64, J=64, Y=a, zq=None, zs=None, st=a):
        return L.bimask_linear_fwd(X, vals, hw, bias, act, R, T, I, J, Y, zq, zs, st, None)

    for kw, word in (({"T": 0}, "T = 0"), ({"T": -3}, "T = -3"), ({"I": 48}, "I = 48"), ({"J": 0}, "J = 0"), ({"act": 5}, "activation 5"),
                     ({"act": -1}, "activation -1"), ({"X": None}, "null"), ({"vals": None}, "null"), ({"Y": None}, "null"),
                     ({"st": None}, "null"), ({"zq": a}, "both"), ({"zs": a}, "both"), ({"X": odd}, "aligned"), ({"bias": odd}, "aligned"),
                     ({"R": odd}, "aligned"), ({"zq": odd, "zs": a}, "aligned"), ({"hw": odd}, "aligned"), ({"Y": odd}, "aligned")):
        assert lin(**kw) == inval and word in bm.bimask_last_error(), (kw, bm.bimask_last_error())

    def bwd(dY=a, zq=a, zs=a, act=2, T=4, C=64, dZ=a, db=a, ws=a, n=1 << 20):
        return L.bimask_act_bwd(dY, zq, zs, act, T, C, dZ, db, ws, n, None)

    for kw, word in (({"T": 0}, "T = 0"), ({"C": 40}, "C = 40"), ({"act": 9}, "activation 9"), ({"dY": None}, "null"),
                     ({"dZ": None, "db": None}, "null"), ({"zq": None}, "slope"), ({"zs": None}, "slope"), ({"ws": None}, "workspace"),
                     ({"n": 8}, "workspace"), ({"dZ": odd}, "aligned"), ({"db": odd}, "aligned"), ({"ws": odd}, "aligned")):
        assert bwd(**kw) == inval and word in bm.bimask_last_error(), (kw, bm.bimask_last_error())

    assert L.bimask_ckpt_pack(a, 0, 64, a, a, None) == inval and L.bimask_ckpt_pack(a, 4, 33, a, a, None) == inval
    assert L.bimask_ckpt_pack(None, 4, 64, a, a, None) == inval and L.bimask_ckpt_pack(a, 4, 64, odd, a, None) == inval
    assert L.bimask_ckpt_unpack(a, a, 7, 4, 64, a, None) == inval and L.bimask_ckpt_unpack(a, None, 0, 4, 64, a, None) == inval
    assert L.bimask_ckpt_unpack(a, a, 0, 4, 64, odd, None) == inval

    def wg(dY=a, q=a, s=a, T=4, I=64, J=64, dW=a, ws=a, n=1 << 24, st=a):
        return L.bimask_wgrad_ckpt(dY, q, s, T, I, J, dW, ws, n, st, None)

    for kw, word in (({"T": 0}, "T = 0"), ({"I": 16}, "I = 16"), ({"J": 65}, "J = 65"), ({"dY": None}, "null"), ({"q": None}, "null"),
                     ({"s": None}, "null"), ({"dW": None}, "null"), ({"ws": None}, "null"), ({"st": None}, "null"), ({"n": 16, "T": 4096}, "workspace"),
                     ({"dW": odd}, "aligned"), ({"s": odd}, "aligned")):
        assert wg(**kw) == inval and word in bm.bimask_last_error(), (kw, bm.bimask_last_error())
    assert bm.bimask_launch_count() == n0
    with pytest.raises(bm.BimaskError, match="activation 6"):
        bm.bimask_ckpt_unpack(a, a, 6, 4, 64, a, stream=0)
    with pytest.raises(ValueError, match="contiguous"):
        bm.bimask_ckpt_pack(torch.zeros(64, 8).t(), 8, 64, a, a, stream=0)
