"""CPU checks of dropout and the residual junction: the plain 64-bit statements against published vectors, autograd and
differences, the size query, and the refusals of the library's entry points (no GPU is touched)."""
import numpy as np
import pytest
import torch

from oracle import residual_oracle as RO


@pytest.fixture(scope="module")
def bm():
    from paper_2302_06058_b200 import build
    build.build()
    import paper_2302_06058_b200 as m
    m.lib()
    return m


def test_generator_gives_the_published_vectors():
    """The known answers that the authors of the generator publish with it (Random123, philox4x32 with 10 rounds)."""
    for counter, key, want in (((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
                               ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
                               ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
                                (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))):
        got = RO.philox([np.array([c]) for c in counter], key)
        assert [int(w[0]) for w in got] == list(want)


@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.9])
def test_share_of_kept_elements(p):
    """A binomial count within five deviations, in every column position of a block and overall; rows do not depend on the batch."""
    T, C = 2000, 64
    k = RO.keep(T, C, p, 77, 5)
    n, thr = T * C, RO.threshold(p)
    for part in (k, *(k[:, i::8] for i in range(8))):
        q = 1 - thr / 65536
        assert abs(part.sum() - part.size * q) <= 5 * np.sqrt(part.size * q * (1 - q)) + 1e-9
    assert np.array_equal(RO.keep(30, C, p, 77, 5, first_row=9), k[9:39])
    if 0 < p < 1:
        other = RO.keep(T, C, p, 77, 6), RO.keep(T, C, p, 78, 5), RO.keep(T, C, p, 77 + (1 << 32), 5)
        same = 1 - 2 * (thr / 65536) * (1 - thr / 65536)                # two independent masks agree with this probability
        for o in other:
            assert abs((o == k).mean() - same) <= 5 * np.sqrt(same * (1 - same) / n)


def test_thresholds():
    assert [RO.threshold(p) for p in (0.0, 2.0 ** -18, 2.0 ** -16, 0.5, 1 - 2.0 ** -20)] == [0, 0, 1, 32768, 65535]


def _problem(rng, T, C, gates):
    r = rng.standard_normal
    return dict(x=2 * r((T, C)) + 0.5, y=r((T, C)) - 0.3, gate=r((gates, C)), scale=r(C), w_post=1 + 0.3 * r(C), b_post=r(C),
                w_pre=1 + 0.3 * r(C), b_pre=r(C))


@pytest.mark.parametrize("post,pre", [(0, 1), (0, 2), (1, 1), (2, 2), (2, 0), (1, 2), (0, 0)])
@pytest.mark.parametrize("span", [0, 1, 3])
def test_gradients_against_autograd_and_differences(post, pre, span):
    rng = np.random.default_rng(10 * post + pre + 100 * span)
    T, C, eps, alpha = 7, 32, 1e-3, 0.7
    q = _problem(rng, T, C, -(-T // max(span, 1)))
    m = RO.multiplier(T, C, 0.3, 5, 6)
    cx, cn = rng.standard_normal((T, C)), rng.standard_normal((T, C))        # the loss is sum(cx x') + sum(cn n)
    kw = dict(post=post, pre=pre, alpha=alpha, span=max(span, 1), m=m, eps_post=eps, eps_pre=2 * eps)
    if not span:
        q["gate"] = None
    if post == RO.NONE:
        q["w_post"] = q["b_post"] = None
    if pre == RO.NONE:
        q["w_pre"] = q["b_pre"] = None

    def loss(v):
        o = RO.forward(v["x"], v["y"], gate=v["gate"], scale=v["scale"], w_post=v["w_post"], b_post=v["b_post"], w_pre=v["w_pre"],
                       b_pre=v["b_pre"], **kw)
        return float((cx * o["xo"]).sum() + (0.0 if o["n"] is None else (cn * o["n"]).sum()))

    f = RO.forward(q["x"], q["y"], gate=q["gate"], scale=q["scale"], w_post=q["w_post"], b_post=q["b_post"], w_pre=q["w_pre"],
                   b_pre=q["b_pre"], **kw)
    bk = {k: v for k, v in kw.items() if not k.startswith("eps")}
    g = RO.backward(cx, cn, f["xo"], q["y"], f["stats_post"], f["stats_pre"], gate=q["gate"], scale=q["scale"], w_post=q["w_post"],
                    b_post=q["b_post"], w_pre=q["w_pre"], **bk)

    t = {k: None if v is None else torch.tensor(v, requires_grad=True) for k, v in q.items()}

    def norm(v, kind, e, w, b):
        v = v - v.mean(1, keepdim=True) if kind == RO.LAYER else v
        return v / torch.sqrt((v * v).mean(1, keepdim=True) + e) * w + b

    u = t["y"] if post == RO.NONE else norm(t["y"], post, eps, t["w_post"], t["b_post"])
    u = u * torch.tensor(m) * t["scale"]
    if span:
        u = u * t["gate"][torch.arange(T) // span]
    xo = alpha * t["x"] + u
    total = (torch.tensor(cx) * xo).sum()
    if pre != RO.NONE:
        total = total + (torch.tensor(cn) * norm(xo, pre, 2 * eps, t["w_pre"], t["b_pre"])).sum()
    total.backward()
    assert abs(float(total.detach()) - loss(q)) < 1e-9 * (1 + abs(loss(q)))
    for k, v in t.items():
        if v is None:
            continue
        assert np.allclose(g["d" + k], v.grad.numpy(), rtol=1e-9, atol=1e-10), k
        for _ in range(6):                                                   # a few entries by central differences
            i = tuple(rng.integers(0, n) for n in q[k].shape)
            h, lo, hi = 1e-5, q[k].copy(), q[k].copy()
            lo[i] -= h
            hi[i] += h
            d = (loss({**q, k: hi}) - loss({**q, k: lo})) / (2 * h)
            assert abs(d - g["d" + k][i]) <= 1e-6 * (1 + abs(d)), (k, i)


def test_workspace_query(bm):
    q = bm.bimask_residual_norm_workspace_bytes
    assert q(0, 64, 1) == q(4, 48, 1) == q(4, 16416, 1) == q(4, 64, 0) == q(-1, 64, 1) == 0
    for C in (32, 384, 1152, 4096, 4128, 8192, 16384):
        for span in (1, 2, 7, 197, 5000):
            sizes = [q(T, C, span) for T in (*range(1, 400), 1000, 2367, 2368, 2369, 4736, 4737, 12608, 16384, 100000, 1 << 30)]
            assert sizes == sorted(sizes) and sizes[0] >= 16 * C


def test_refusals_name_the_cause(bm):
    """Every bad argument is refused on the host, before any launch."""
    L, inval = bm.lib(), bm.binding.BIMASK_EINVAL
    n0 = bm.bimask_launch_count()
    a, odd = 256, 264                                       # addresses that are never dereferenced: aligned, misaligned

    def drop(X=a, type=0, T=4, C=64, d=bm.make_dropout(0.1, 1), Y=a):
        return L.bimask_dropout(X, type, T, C, d, Y, None)

    bad_p = [({"d": bm.make_dropout(p, 1)}, "p = ") for p in (-0.1, 1.0, 1.5, float("nan"))]
    for kw, word in (({"T": 0}, "T = 0"), ({"C": 40}, "C = 40"), ({"type": 2}, "type 2"), ({"d": None}, "null"), ({"X": None}, "null"), ({"Y": None}, "null"),
                     ({"X": odd}, "aligned"), ({"Y": odd}, "aligned"), ({"d": bm.make_dropout(0.1, 1, 0, 260)}, "counter"), *bad_p):
        assert drop(**kw) == inval and word in bm.bimask_last_error(), (kw, bm.bimask_last_error())

    def unpack(q=a, s=a, act=2, d=bm.make_dropout(0.1, 1), T=4, C=64, X=a):
        return L.bimask_ckpt_unpack_dropout(q, s, act, d, T, C, X, None)

    for kw, word in (({"T": -1}, "T = -1"), ({"C": 0}, "C = 0"), ({"act": 5}, "activation 5"), ({"q": None}, "null"), ({"s": odd}, "aligned"), ({"d": None}, "null"),
                     *bad_p):
        assert unpack(**kw) == inval and word in bm.bimask_last_error(), (kw, bm.bimask_last_error())

    def bwd(dY=a, zq=a, zs=a, act=2, d=bm.make_dropout(0.1, 1), T=4, C=64, dZ=a, db=a, ws=a, n=1 << 20):
        return L.bimask_act_dropout_bwd(dY, zq, zs, act, d, T, C, dZ, db, ws, n, None)

    for kw, word in (({"T": 0}, "T = 0"), ({"C": 40}, "C = 40"), ({"act": -1}, "activation -1"), ({"dZ": None, "db": None}, "null"), ({"zq": None}, "slope"),
                     ({"n": 8}, "workspace"), ({"dY": odd}, "aligned"), ({"d": None}, "null"), *bad_p):
        assert bwd(**kw) == inval and word in bm.bimask_last_error(), (kw, bm.bimask_last_error())

    def args(T=4, C=64, post=1, pre=2, drop=bm.make_dropout(0.1, 1), span=2, pitch=None, eps=1e-5, alpha=1.0, type=0, without=(), **kw):
        b = {k: a for k in bm.binding._RESIDUAL_POINTERS}
        b.update({"ws_bytes": 1 << 24, **kw})
        for k in without:
            b[k] = None
        r = bm.make_residual_args(T, C, b, type, post, pre, eps, eps, alpha, span, drop)
        if pitch is not None:
            r.gate_pitch = pitch
        return r

    unsupported = bm.binding.BIMASK_EUNSUPPORTED
    both = (L.bimask_residual_norm_fwd, L.bimask_residual_norm_bwd)
    nan, inf = float("nan"), float("inf")
    for kw, word in (({"T": 0}, "T = 0"), ({"T": -5}, "T = -5"), ({"C": 48}, "C = 48"), ({"type": 3}, "type 3"), ({"post": 3}, "norm 3"), ({"pre": -1}, "norm"),
                     ({"eps": -1.0}, "eps"), ({"eps": nan}, "eps"), ({"alpha": inf}, "alpha"), ({"drop": bm.make_dropout(1.0, 1)}, "p = 1"),
                     ({"drop": bm.make_dropout(0.1, 1, 0, 4)}, "counter"), ({"span": 0}, "gate_span"), ({"pitch": 56}, "gate_pitch"), ({"pitch": 68}, "gate_pitch"),
                     ({"post": 0}, "without their norm"), ({"pre": 0}, "without their norm"),
                     *(({k: odd}, "aligned") for k in bm.binding._RESIDUAL_POINTERS)):
        for call in both:
            assert call(args(**kw), None) == inval and word in bm.bimask_last_error(), (kw, bm.bimask_last_error())
    for call in both:
        assert call(args(C=16416), None) == unsupported and "16384" in bm.bimask_last_error()
        assert call(None, None) == inval
    fwd, bwd_ = both
    no_w = ("w_post", "b_post")
    for kw, word in (({"without": ("x",)}, "null"), ({"without": ("n",)}, "null"), ({"pre": 0, "without": ("xo", "w_pre", "b_pre")}, "null"),
                     ({"without": ("y",)}, "without a branch"), ({"post": 0, "without": ("y", "gate", "scale", *no_w)}, "without a branch")):
        assert fwd(args(**kw), None) == inval and word in bm.bimask_last_error(), (kw, bm.bimask_last_error())
    grads = ("dx", "dy", "dgate", "dscale", "dw_post", "db_post", "dw_pre", "db_pre")
    for kw, word in (({"without": ("dn",)}, "null"), ({"without": ("xo",)}, "null"), ({"without": ("stats_pre",)}, "null"), ({"without": ("stats_post",)}, "stats_post"),
                     ({"pre": 0, "without": ("w_pre", "b_pre", "dxo", "dw_pre", "db_pre")}, "null"), ({"pre": 0, "without": ("w_pre", "b_pre")}, "absent"),
                     ({"post": 0, "without": no_w}, "absent"), ({"without": grads}, "no gradient"), ({"without": ("gate",)}, "gate"), ({"without": ("y",)}, "y is needed"),
                     ({"without": ("ws",)}, "workspace"), ({"ws_bytes": 512}, "workspace"),
                     ({"post": 0, "without": ("y", "gate", "scale", *no_w, *grads[1:6])}, "without a branch")):
        assert bwd_(args(**kw), None) == inval and word in bm.bimask_last_error(), (kw, bm.bimask_last_error())
    assert bm.bimask_launch_count() == n0
    with pytest.raises(bm.BimaskError, match="gate_span"):
        bm.bimask_residual_norm_fwd(args(span=0), stream=0)
    with pytest.raises(ValueError, match="contiguous"):
        bm.make_residual_args(4, 64, {"y": torch.zeros(64, 4).t()})
    with pytest.raises(ValueError, match="contiguous"):
        bm.make_residual_args(4, 64, {"gate": torch.zeros(64, 4).t()})
    with pytest.raises(ValueError, match="pitch"):
        bm.make_residual_args(4, 64, {"gate": torch.zeros(4, 128)[:, :64], "dgate": torch.zeros(4, 64)})
