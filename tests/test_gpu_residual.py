"""The residual junction and its gradient on the GPU against their plain 64-bit statements.

Tolerances, derived before the first run.  u = 2^-24 is half a step of fp32.  A value that is put together by sums and products
along at most n roundings is off by at most n u times the same expression with every term replaced by its magnitude (first
order).  The longest paths: a row's sum takes 8 additions in a thread, 1 + 5 + 4 across lanes and warps and 3 products (21); a
normalised value two roundings more, and an affine map, gate, scale and dropout 6: 32 per norm; a backward pass through both norms 64.
Magnitude of a normalised value: (|v| + mean |v|) rstd.  The relative error of a computed rstd: half that of the sum of squares of
d = v - mean, each off by 24 u (|v| + mean |v|): at most 32 u (1 + max (|v| + mean |v|) rstd).  A bf16 result must lie between the
roundings of want - tolerance and want + tolerance.  Sums over tokens: T + 64 roundings."""
import itertools

import numpy as np
import pytest
import torch

import paper_2302_06058_b200 as bm
from oracle import residual_oracle as RO

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SEED, NUMBER = 0x1234567890ABCDEF, 77
EPS = (1e-5, 1e-6)
TYPES = {"bf16": (torch.bfloat16, bm.TYPE_BF16), "f32": (torch.float32, bm.TYPE_F32)}


def r(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a)).float().to(dtype)


def between(got, want, tol):
    """Element-wise: got lies between want - tol and want + tol, rounded to its type."""
    g = got.double().cpu().numpy()
    if got.dtype == torch.float32:
        return np.abs(g - want) <= tol + U * np.abs(want)
    return (r(want - tol, got.dtype).double().numpy() <= g) & (g <= r(want + tol, got.dtype).double().numpy())


def check(name, got, want, tol):
    ok = between(got, want, tol)
    assert ok.all(), (name, int((~ok).sum()), np.argwhere(~ok)[:3].tolist(), float(np.abs(got.double().cpu().numpy() - want).max()))


class Problem:
    """Random inputs of one junction, on the device and in 64 bits."""

    def __init__(self, T, C, post, pre, stream="bf16", span=0, scale=True, bias=True, p=0.0, alpha=1.0, seed=1, offset=0.0, pitch=None):
        rng = np.random.default_rng(seed + T * 31 + C)
        self.T, self.C, self.post, self.pre, self.span, self.p, self.alpha = T, C, post, pre, span, p, float(np.float32(alpha))
        self.dt, self.code = TYPES[stream]
        self.h, self.d = {}, {}                            # 64-bit host copies, device tensors
        bf = torch.bfloat16

        def put(k, a, dt):
            t = r(a, dt)
            self.d[k], self.h[k] = t.cuda(), t.double().numpy()

        def rows(s=1.0):
            a = rng.standard_normal((T, C)) * s
            a[:, ::64] *= 8
            return a

        put("x", rows(2.0) + offset, self.dt)
        put("y", rows(0.5) + offset, bf)
        put("dxo", rows(0.01), self.dt)
        put("dn", rows(0.01), bf)
        if span:
            n = -(-T // span)
            wide = np.zeros((n, pitch or C))
            wide[:, :C] = rng.standard_normal((n, C))
            put("gate", wide, bf)
            if pitch:
                self.wide = self.d["gate"]
                self.d["gate"] = self.wide[:, :C]
                self.h["gate"] = self.h["gate"][:, :C]
        if scale:
            put("scale", 0.1 + rng.random(C), torch.float32)
        for side, kind in (("post", post), ("pre", pre)):
            if kind:
                put("w_" + side, 1 + 0.3 * rng.standard_normal(C), torch.float32)
                if bias:
                    put("b_" + side, 0.3 * rng.standard_normal(C), torch.float32)
        self.m = RO.multiplier(T, C, p, SEED, NUMBER)
        self.drop = bm.make_dropout(p, SEED, NUMBER)

    def like(self, **kw):
        return {k: torch.full(shape, 7.0, dtype=dt, device="cuda") for k, (shape, dt) in kw.items()}

    def args(self, bufs):
        return bm.make_residual_args(self.T, self.C, bufs, self.code, self.post, self.pre, *EPS, self.alpha, max(self.span, 1), self.drop)

    def outputs(self):
        s, f = (self.T, self.C), torch.float32
        o = self.like(xo=(s, self.dt))
        for side, kind in (("post", self.post), ("pre", self.pre)):
            if kind:
                o.update(self.like(**{"stats_" + side: ((self.T, 2), f)}))
        if self.pre:
            o.update(self.like(n=(s, torch.bfloat16)))
        return o

    def gradients(self):
        s, f, c = (self.T, self.C), torch.float32, (self.C,)
        g = self.like(dx=(s, self.dt), dy=(s, torch.bfloat16))
        for k in ("scale", "w_post", "b_post", "w_pre", "b_pre"):
            if k in self.d:
                g.update(self.like(**{"d" + k: (c, f)}))
        if self.span:
            g["dgate"] = torch.full_like(self.wide, 7.0)[:, :self.C] if hasattr(self, "wide") else torch.full_like(self.d["gate"], 7.0)
        g["ws"] = torch.full((bm.bimask_residual_norm_workspace_bytes(self.T, self.C, max(self.span, 1)),), 0xFF, dtype=torch.uint8, device="cuda")
        return g

    def pick(self, *names):
        return {k: self.d[k] for k in names if k in self.d}

    def forward(self, **override):
        o = self.outputs()
        o.update(override)
        bm.bimask_residual_norm_fwd(self.args({**self.pick("x", "y", "gate", "scale", "w_post", "b_post", "w_pre", "b_pre"), **o}))
        return o

    def backward(self, f, **override):
        g = self.gradients()
        g.update(override)
        bufs = {**self.pick("dxo", "y", "gate", "scale", "w_post", "b_post", "w_pre"), **g}
        if self.pre:
            bufs.update(dn=self.d["dn"], xo=f["xo"], stats_pre=f["stats_pre"])
        if self.post:
            bufs["stats_post"] = f["stats_post"]
        bm.bimask_residual_norm_bwd(self.args(bufs))
        return g

    # the statements and their tolerances
    def hat_tolerance(self, v, hat, rstd, extra=0.0):
        """(of the normalised values, relative of rstd) where v itself is off by up to `extra`."""
        extra = np.broadcast_to(extra, v.shape)
        mag = (np.abs(v) + np.abs(v).mean(1, keepdims=True)) * rstd
        rel = 32 * U * (1 + mag.max(1, keepdims=True)) + 2 * (extra * rstd).max(1, keepdims=True)
        return 32 * U * mag + (extra + extra.mean(1, keepdims=True)) * rstd + np.abs(hat) * rel, rel

    def check_forward(self, o):
        h, span = self.h, max(self.span, 1)
        w = RO.forward(h["x"], h["y"], self.post, self.pre, float(np.float32(EPS[0])), float(np.float32(EPS[1])), self.alpha, h.get("gate"), span,
                       h.get("scale"), self.m, h.get("w_post"), h.get("b_post"), h.get("w_pre"), h.get("b_pre"))
        g, s = RO.gate_rows(h.get("gate"), span, self.T), h.get("scale", 1.0)
        factor = np.abs(s * g * self.m)
        u, du = np.abs(h["y"]), 0.0
        if self.post:
            st = w["stats_post"]
            hat = RO.normalised(h["y"], st)
            t, rel = self.hat_tolerance(h["y"], hat, st[:, 1:])
            du = t * np.abs(h["w_post"])
            u = np.abs(hat * h["w_post"]) + np.abs(h.get("b_post", 0.0))
            check("mean", o["stats_post"][:, :1], st[:, :1], 32 * U * np.abs(h["y"]).mean(1, keepdims=True))
            check("rstd", o["stats_post"][:, 1:], st[:, 1:], rel * st[:, 1:])
        tx = factor * (du + 8 * U * u) + 2 * U * np.abs(self.alpha * h["x"])
        check("xo", o["xo"], w["xo"], tx)
        if self.pre:
            st = w["stats_pre"]
            hat = RO.normalised(w["xo"], st)
            t, rel = self.hat_tolerance(w["xo"], hat, st[:, 1:], tx)
            check("mean", o["stats_pre"][:, :1], st[:, :1], 32 * U * np.abs(w["xo"]).mean(1, keepdims=True) + tx.mean(1, keepdims=True))
            check("rstd", o["stats_pre"][:, 1:], st[:, 1:], rel * st[:, 1:])
            check("n", o["n"], w["n"], t * np.abs(h["w_pre"]) + 4 * U * (np.abs(hat * h["w_pre"]) + np.abs(h.get("b_pre", 0.0))))

    def check_backward(self, g, f, only=None):
        h, span = self.h, max(self.span, 1)
        xo = f["xo"].double().cpu().numpy()
        sp = f["stats_post"].double().cpu().numpy() if self.post else None
        sn = f["stats_pre"].double().cpu().numpy() if self.pre else None
        kw = dict(post=self.post, pre=self.pre, alpha=self.alpha, gate=h.get("gate"), span=span, scale=h.get("scale"), w_post=h.get("w_post"),
                  b_post=h.get("b_post"), w_pre=h.get("w_pre"))
        want = RO.backward(h["dxo"], h["dn"], xo, h["y"], sp, sn, m=self.m, **kw)
        # the same expressions in magnitudes
        a = {k: np.abs(v) if isinstance(v, np.ndarray) else v for k, v in kw.items()}
        mag = self.magnitudes(a, xo, sp, sn, span)
        for k in want:
            if k in g and (only is None or k in only):
                n = 64 + (self.T if want[k].ndim == 1 else span if k == "dgate" else 0)
                check(k, g[k], want[k], n * U * mag[k])

    def magnitudes(self, a, xo, sp, sn, span):
        h, out = self.h, {}

        def hat(v, st):
            return (np.abs(v) + np.abs(st[:, :1])) * st[:, 1:]

        def through(g, x, rstd):
            return rstd * (g + g.mean(1, keepdims=True) + x * (g * x).mean(1, keepdims=True))

        D = np.abs(h["dxo"])
        if self.pre:
            x, dn = hat(xo, sn), np.abs(h["dn"])
            out["dw_pre"], out["db_pre"] = (dn * x).sum(0), dn.sum(0)
            D = D + through(dn * RO._or(a["w_pre"], 1.0), x, sn[:, 1:])
        out["dx"] = abs(self.alpha) * D
        g, s = RO.gate_rows(a["gate"], span, self.T), RO._or(a["scale"], 1.0)
        y = hat(h["y"], sp) if self.post else np.abs(h["y"])
        u = y * RO._or(a["w_post"], 1.0) + RO._or(a["b_post"], 0.0)
        if a["gate"] is not None:
            out["dgate"] = np.add.reduceat(D * s * self.m * u, np.arange(0, self.T, span), axis=0)
        out["dscale"] = (D * g * self.m * u).sum(0)
        du = D * s * g * self.m
        if self.post:
            out["dw_post"], out["db_post"] = (du * y).sum(0), du.sum(0)
            du = through(du * RO._or(a["w_post"], 1.0), y, sp[:, 1:])
        out["dy"] = du
        return out


# one token, a few, several rows per group; one warp, parts of one, several, the widest rows of one, two and four CTAs; as many rows
# as one CTA's launch takes in the backward pass, and one more
SIZES = [(1, 32), (3, 64), (2, 256), (32, 256), (33, 256), (37, 288), (5, 512), (70, 544), (301, 384), (33, 1152), (6, 2080), (4, 4096), (3, 4128), (5, 8192), (3, 8224), (9, 16384)]
FORMS = [(0, 1), (0, 2), (1, 1), (2, 2), (1, 2), (2, 1), (1, 0), (2, 0), (0, 0)]


@pytest.mark.parametrize("T,C", SIZES)
@pytest.mark.parametrize("stream", TYPES)
def test_against_64_bits(T, C, stream):
    for i, ((post, pre), k) in enumerate(itertools.product(FORMS, range(5 if C < 600 else 1))):
        span = (0, 1, 2, T, T + 3)[k if C < 600 else i % 5]
        q = Problem(T, C, post, pre, stream, span=span, scale=i % 2 == 0, bias=i % 3 != 0, p=(0.0, 0.3)[(i // 2) % 2], alpha=(1.0, 0.8)[i % 2])
        f = q.forward()
        q.check_forward(f)
        g = q.backward(f)
        q.check_backward(g, f)
        f2, g2 = q.forward(), q.backward(f)                                # and the same bits again
        assert all(torch.equal(f[k], f2[k]) for k in f) and all(torch.equal(g[k], g2[k]) for k in g if k != "ws")


# widths whose backward pass takes one row per step in some forms: rows of three, five, six, nine and twelve warps, and the first that
# two CTAs share again; as many rows as one CTA's launch takes and one more, and more than one row per group of warps
ONE_ROW = [(8, 1152), (9, 1152), (650, 1056), (4, 2080), (5, 2560), (310, 2336), (3, 2816), (2, 4128), (3, 4608), (301, 5120), (160, 6144), (40, 6176)]


@pytest.mark.parametrize("T,C", ONE_ROW)
@pytest.mark.parametrize("stream", TYPES)
def test_widths_of_one_row_per_step(T, C, stream):
    for i, (post, pre) in enumerate([(0, 1), (0, 2), (1, 1), (1, 2), (1, 0), (0, 0)]):
        q = Problem(T, C, post, pre, stream, span=(0, 1, 2, T)[(i + T) % 4], scale=i % 2 == 1, bias=i % 3 == 1, p=(0.3, 0.0)[i // 3], alpha=(0.8, 1.0)[i % 2])
        f = q.forward()
        g = q.backward(f)
        q.check_backward(g, f)
        g2 = q.backward(f)                                                 # and the same bits again
        assert all(torch.equal(g[k], g2[k]) for k in g if k != "ws")


@pytest.mark.parametrize("T,C", [(1, 32), (24, 256), (25, 256), (1800, 384), (12, 768), (13, 768), (601, 1024), (4, 2048), (155, 3584), (301, 4096)])
@pytest.mark.parametrize("stream", TYPES)
def test_a_gate_per_token_with_means_or_biases(T, C, stream):
    for post, pre in ((0, 2), (0, 1), (2, 1)):
        q = Problem(T, C, post, pre, stream, span=1, scale=pre == 1, p=0.2)
        f = q.forward()
        g = q.backward(f)
        q.check_backward(g, f)
        for k in ("dgate", "dscale", "dw_pre", "dy"):                      # every gradient alone is what it is among the others
            if k in g:
                alone = q.backward(f, **{o: None for o in g if o not in (k, "ws")})
                assert torch.equal(alone[k], g[k]), k


@pytest.mark.parametrize("T,C,span", [(900, 1152, 5), (700, 1536, 350), (500, 2560, 97), (400, 5120, 6), (300, 6144, 1000), (310, 4608, 2)])
@pytest.mark.parametrize("stream", TYPES)
def test_widths_of_one_row_per_step_and_gates_that_serve_spans(T, C, span, stream):
    for post, pre in ((0, 2), (1, 1), (1, 0)):
        q = Problem(T, C, post, pre, stream, span=span, bias=post == 0, p=0.1)
        f = q.forward()
        q.check_backward(q.backward(f), f)


@pytest.mark.parametrize("T,C,span", [(2500, 256, 7), (2500, 64, 1300), (700, 1152, 197), (4000, 320, 3999), (300, 4160, 2), (149, 4096, 150), (9000, 64, 7), (600, 8192, 64), (200, 9216, 200)])
def test_many_rows_and_gates_that_serve_spans(T, C, span):
    """More rows than groups of warps: units of several rows, spans that end inside and a last span that is not full."""
    for post, pre in ((0, 2), (1, 1), (2, 0)):
        q = Problem(T, C, post, pre, span=span, p=0.1)
        f = q.forward()
        q.check_forward(f)
        q.check_backward(q.backward(f), f)


@pytest.mark.parametrize("post,pre", [(2, 2), (1, 1)])
def test_rows_far_from_zero_and_constant_rows(post, pre):
    """A mean a thousand deviations from zero (the tolerance grows with it, as the inputs' own rounding does), rows without any
    deviation and rows of zeros: eps decides."""
    q = Problem(20, 416, post, pre, "f32", offset=1000.0, p=0.2)
    f = q.forward()
    q.check_forward(f)
    q.check_backward(q.backward(f), f)
    q = Problem(6, 96, post, pre, "f32", scale=False)
    for k in ("x", "y"):
        for row, v in ((0, 0.0), (1, 0.0), (2, 3.0)):
            q.d[k][row] = v
            q.h[k][row] = v
    f = q.forward()
    q.check_forward(f)
    q.check_backward(q.backward(f), f)


@pytest.mark.parametrize("stream", TYPES)
def test_parts_that_are_absent(stream):
    """The norm alone (first block), the last junction without a norm, gradients from one side only, single gradients."""
    T, C = 45, 288
    for pre, alpha in ((1, 1.0), (2, 0.5)):
        q = Problem(T, C, 0, pre, stream, scale=False, alpha=alpha)
        o = q.outputs()
        a = {**q.pick("x", "w_pre", "b_pre"), **o}
        bm.bimask_residual_norm_fwd(q.args(a))
        h = q.h
        w = RO.forward(h["x"], None, 0, pre, 0, float(np.float32(EPS[1])), alpha, w_pre=h["w_pre"], b_pre=h["b_pre"])
        check("xo", o["xo"], w["xo"], U * np.abs(w["xo"]))
        t, _ = q.hat_tolerance(w["xo"], RO.normalised(w["xo"], w["stats_pre"]), w["stats_pre"][:, 1:])
        check("n", o["n"], w["n"], t * np.abs(h["w_pre"]) + 4 * U * (np.abs(w["n"]) + 2 * np.abs(h["b_pre"])))
        n2 = torch.empty_like(o["n"])
        bm.bimask_residual_norm_fwd(q.args({**q.pick("x", "w_pre", "b_pre"), "n": n2}))           # n alone
        assert torch.equal(n2, o["n"])
        g = q.gradients()
        bm.bimask_residual_norm_bwd(q.args({"dn": q.d["dn"], "w_pre": q.d["w_pre"], "xo": o["xo"], "stats_pre": o["stats_pre"],
                                            **{k: g[k] for k in ("dx", "dw_pre", "db_pre", "ws")}}))
        xo, st = o["xo"].double().cpu().numpy(), o["stats_pre"].double().cpu().numpy()
        want = RO.backward(None, h["dn"], xo, None, None, st, pre=pre, alpha=alpha, w_pre=h["w_pre"])
        q.h["dxo"] = np.zeros((T, C))
        mag = q.magnitudes(dict(w_pre=np.abs(h["w_pre"]), gate=None, scale=None, w_post=None, b_post=None), xo, None, st, 1)
        for k in ("dx", "dw_pre", "db_pre"):
            check(k, g[k], want[k], (64 + (T if k != "dx" else 0)) * U * mag[k])
    # no parameters at all, and plain residual addition, whose gradient does not read y
    q = Problem(T, C, 0, 0, stream, scale=False, p=0.4)
    f = q.forward()
    q.check_forward(f)
    g = q.gradients()
    bm.bimask_residual_norm_bwd(q.args({"dxo": q.d["dxo"], "dx": g["dx"], "dy": g["dy"]}))
    q.check_backward({k: g[k] for k in ("dx", "dy")}, f)
    q = Problem(T, C, 2, 2, stream, span=9, p=0.1)
    for k in ("w_post", "b_post", "w_pre", "b_pre", "scale"):
        del q.d[k]
        q.h[k] = np.full(C, float(k[0] != "b"))
    f = q.forward()
    q.check_forward(f)
    g = q.backward(f)
    q.check_backward({k: g[k] for k in ("dx", "dy", "dgate")}, f)
    # gradients of a scale and a weight that are absent in the forward pass, and so 1
    for post in (0, 2):
        q = Problem(T, C, post, 1, stream, span=1, p=0.1)
        for k in ("w_post", "scale"):
            if k in q.d:
                del q.d[k]
                q.h[k] = np.ones(C)
        f = q.forward()
        more = q.like(dscale=((C,), torch.float32), **({"dw_post": ((C,), torch.float32)} if post else {}))
        q.check_backward(q.backward(f, **more), f)
    # every gradient alone is what it is among the others
    q = Problem(T, C, 2, 2, stream, span=9, p=0.1)
    f = q.forward()
    g = q.backward(f)
    for k in g:
        if k != "ws":
            alone = q.backward(f, **{o: None for o in g if o not in (k, "ws")})
            assert torch.equal(alone[k], g[k]), k


@pytest.mark.parametrize("stream", TYPES)
@pytest.mark.parametrize("T,C", [(50, 320), (9, 4224), (700, 4128)])
def test_results_in_the_place_of_inputs(T, C, stream):
    for post, pre in ((1, 1), (2, 2), (0, 2)):
        q = Problem(T, C, post, pre, stream, span=1, p=0.1)
        f = q.forward()
        g = q.backward(f)
        x, y = q.d["x"].clone(), q.d["y"].clone()
        keep_x, keep_y = q.d["x"], q.d["y"]
        q.d["x"], q.d["y"] = x, y
        o = q.forward(xo=x, n=y)
        assert torch.equal(o["xo"], f["xo"]) and torch.equal(o["n"], f["n"])
        q.d["x"], q.d["y"] = keep_x, keep_y
        for target in ("dn", "y"):
            saved = {k: q.d[k].clone() for k in ("dxo", target)}
            i = q.backward(f, dx=q.d["dxo"], dy=q.d[target])
            assert all(torch.equal(i[k], g[k]) for k in g if k != "ws")
            q.d.update(saved)


@pytest.mark.parametrize("span", [1, 5])
def test_gate_rows_of_a_wider_matrix_and_nothing_outside_the_results(span):
    T, C, pitch, pad = 23, 160, 480, 4096
    q = Problem(T, C, 1, 2, span=span, p=0.1, pitch=pitch)
    guards = []

    def guarded(like):
        n = like.numel()
        b = torch.full((n + 2 * pad,), 7.0, device="cuda").to(like.dtype)
        guards.append((b, n))
        return b[pad:pad + n].view(like.shape)

    f = q.forward(**{k: guarded(v) for k, v in q.outputs().items()})
    q.check_forward(f)
    g0 = q.gradients()
    g = q.backward(f, **{k: guarded(v) for k, v in g0.items() if k not in ("dgate", "ws")}, dgate=g0["dgate"], ws=guarded(g0["ws"]))
    q.check_backward(g, f)
    torch.cuda.synchronize()
    for b, n in guards:
        assert bool((b[:pad] == 7.0).all()) and bool((b[pad + n:] == 7.0).all())
    rest = g0["dgate"]._base[:, C:] if g0["dgate"]._base is not None else None
    assert rest is not None and bool((rest == 7.0).all())


@pytest.mark.parametrize("post,pre", [(1, 1), (2, 2)])
def test_what_is_not_finite_stays_in_its_row(post, pre):
    T, C = 40, 544
    q = Problem(T, C, post, pre, p=0.1)
    for row, v in ((3, float("nan")), (17, float("inf"))):
        q.d["y"][row, 5] = v
    q.d["x"][30, 7] = float("nan")
    f = q.forward()
    fine = torch.ones(T, dtype=torch.bool)
    fine[[3, 17, 30]] = False
    for k in ("xo", "n"):
        assert bool(torch.isfinite(f[k].float()[fine.cuda()]).all())
        assert not bool(torch.isfinite(f[k].float()[~fine.cuda()]).all(1).any())
    g = q.backward(f)
    for k in ("dx", "dy"):
        assert bool(torch.isfinite(g[k].float()[fine.cuda()]).all()), k


def test_captured_passes_that_share_a_workspace():
    """Two junctions' forward and backward passes captured into a graph each, replayed in turn, one workspace between them and a
    counter that moves the masks on."""
    counter = torch.zeros(1, dtype=torch.int64, device="cuda")
    qs = [Problem(120, 384, 0, 2, span=20, p=0.2, seed=3), Problem(64, 1152, 1, 1, p=0.2, seed=4)]
    ws = torch.empty(max(bm.bimask_residual_norm_workspace_bytes(q.T, q.C, max(q.span, 1)) for q in qs), dtype=torch.uint8, device="cuda")
    held, graphs = [], []
    for q in qs:
        q.drop = bm.make_dropout(q.p, SEED, NUMBER, counter)
        f = q.forward()
        held.append((f, q.backward(f, ws=ws)))
    torch.cuda.synchronize()
    for q, (f, g) in zip(qs, held):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            q.forward(**f)
            q.backward(f, **g)
        graphs.append(graph)
    for step in (0, 3):
        counter.fill_(step)
        for i in (0, 1, 0):
            graphs[i].replay()
        torch.cuda.synchronize()
        for q, (f, g) in zip(qs, held):
            q.m = RO.multiplier(q.T, q.C, q.p, SEED, NUMBER + step)
            q.check_forward(f)
            q.check_backward(g, f)


def test_steps_of_a_counter_reach_the_gradient():
    """Forward and backward passes of one step share a mask, those of two steps do not."""
    q = Problem(50, 96, 1, 2, p=0.4)
    counter = torch.zeros(1, dtype=torch.int64, device="cuda")
    q.drop = bm.make_dropout(q.p, SEED, NUMBER - 3, counter)
    seen = []
    for step in (3, 4):
        counter.fill_(step)
        q.m = RO.multiplier(q.T, q.C, q.p, SEED, NUMBER - 3 + step)
        f = q.forward()
        q.check_forward(f)
        g = q.backward(f)
        q.check_backward(g, f)
        seen.append(g["dy"])
    assert not torch.equal(*seen)


def test_another_stream():
    q = Problem(90, 384, 1, 2, p=0.1)
    f = q.forward()
    torch.cuda.synchronize()
    side, o = torch.cuda.Stream(), q.outputs()
    torch.cuda.synchronize()
    bm.bimask_residual_norm_fwd(q.args({**q.pick("x", "y", "scale", "w_post", "b_post", "w_pre", "b_pre"), **o}), stream=side)
    side.synchronize()
    assert all(torch.equal(o[k], f[k]) for k in o)


def test_more_than_2_31_elements():
    """Rows past element 2^31 of every matrix, in place (x' over x, n over y), their masks among them."""
    C = 8192
    T = (1 << 31) // C + 3
    x = torch.zeros(T, C, dtype=torch.bfloat16, device="cuda")
    y = torch.zeros(T, C, dtype=torch.bfloat16, device="cuda")
    q = Problem(4, C, 0, 1, p=0.2, scale=False, bias=False)
    x[-4:], y[-4:] = q.d["x"], q.d["y"]
    q.m = RO.multiplier(4, C, q.p, SEED, NUMBER, first_row=T - 4)
    stats = torch.empty(T, 2, device="cuda")
    a = bm.make_residual_args(T, C, {"x": x, "y": y, "w_pre": q.d["w_pre"], "xo": x, "n": y, "stats_pre": stats}, q.code, 0, 1, *EPS, 1.0, 1, q.drop)
    bm.bimask_residual_norm_fwd(a)
    f = {"xo": x[-4:], "n": y[-4:], "stats_pre": stats[-4:]}
    q.check_forward(f)
    assert not bool(x[:-4].any()) and not bool(y[:-4].any())
    y[-4:] = q.d["y"]
    dn = torch.zeros_like(y)
    dn[-4:] = q.d["dn"]
    dw, ws = torch.empty(C, device="cuda"), torch.empty(bm.bimask_residual_norm_workspace_bytes(T, C, 1), dtype=torch.uint8, device="cuda")
    dx = torch.empty_like(x)
    a = bm.make_residual_args(T, C, {"dn": dn, "xo": x, "stats_pre": stats, "w_pre": q.d["w_pre"], "dx": dx, "dy": dn, "dw_pre": dw, "ws": ws},
                              q.code, 0, 1, *EPS, 1.0, 1, q.drop)
    bm.bimask_residual_norm_bwd(a)
    q.h["dxo"] = np.zeros((4, C))
    q.check_backward({"dx": dx[-4:], "dy": dn[-4:], "dw_pre": dw}, f)
