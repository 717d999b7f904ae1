"""Plain 64-bit statements of what lies between the layers of a transformer block: dropout from a counter-based generator, and
the residual junction (norm after a block, dropout, gate, residual scale, norm before the next) with its gradient.  numpy, one
formula after the other."""
from __future__ import annotations

import numpy as np

NONE, RMS, LAYER = 0, 1, 2


def philox(counter, key):
    """Philox4x32-10 (Salmon, Moraes, Dror, Shaw, SC 2011): counter, 4 arrays of 32-bit words; key, 2 words."""
    low = np.uint64(0xFFFFFFFF)
    c = [np.asarray(w, dtype=np.uint64) for w in counter]
    k = [int(w) for w in key]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def threshold(p):
    return min(65535, int(np.rint(65536.0 * float(np.float32(p)))))


def keep(T, C, p, seed, number, first_row=0):
    """Boolean T x C: which elements of rows first_row .. first_row + T - 1 stay."""
    block = np.arange(first_row * C // 8, (first_row + T) * C // 8, dtype=np.uint64)
    n = np.full_like(block, number & 0xFFFFFFFF), np.full_like(block, (number >> 32) & 0xFFFFFFFF)
    words = philox((block & np.uint64(0xFFFFFFFF), block >> np.uint64(32), *n), (seed & 0xFFFFFFFF, seed >> 32))
    halves = [h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))]
    return (np.stack(halves, -1) >= threshold(p)).reshape(T, C)


def multiplier(T, C, p, seed, number, first_row=0):
    thr = threshold(p)
    return np.ones((T, C)) if thr == 0 else keep(T, C, p, seed, number, first_row) * (65536.0 / (65536 - thr))


def statistics(v, kind, eps):
    """T x 2: mean and 1 / deviation."""
    mean = v.mean(1, keepdims=True) if kind == LAYER else np.zeros((len(v), 1))
    return np.concatenate([mean, 1.0 / np.sqrt(((v - mean) ** 2).mean(1, keepdims=True) + eps)], 1)


def normalised(v, stats):
    return (v - stats[:, :1]) * stats[:, 1:]


def _or(a, default):
    return default if a is None else a


def gate_rows(gate, span, T):
    return 1.0 if gate is None else gate[np.arange(T) // span]


def forward(x, y, post=NONE, pre=NONE, eps_post=0.0, eps_pre=0.0, alpha=1.0, gate=None, span=1, scale=None, m=1.0, w_post=None,
            b_post=None, w_pre=None, b_pre=None):
    """dict of xo, n, stats_post, stats_pre (None where absent)."""
    out = dict(n=None, stats_post=None, stats_pre=None)
    xo = alpha * x
    if y is not None:
        u = y
        if post != NONE:
            out["stats_post"] = statistics(y, post, eps_post)
            u = normalised(y, out["stats_post"]) * _or(w_post, 1.0) + _or(b_post, 0.0)
        xo = xo + _or(scale, 1.0) * gate_rows(gate, span, len(x)) * m * u
    out["xo"] = xo
    if pre != NONE:
        out["stats_pre"] = statistics(xo, pre, eps_pre)
        out["n"] = normalised(xo, out["stats_pre"]) * _or(w_pre, 1.0) + _or(b_pre, 0.0)
    return out


def _through(g, hat, rstd, kind):
    return rstd * (g - (g.mean(1, keepdims=True) if kind == LAYER else 0.0) - hat * (g * hat).mean(1, keepdims=True))


def backward(dxo, dn, xo, y, stats_post, stats_pre, post=NONE, pre=NONE, alpha=1.0, gate=None, span=1, scale=None, m=1.0, w_post=None,
             b_post=None, w_pre=None):
    """Every gradient, given the statistics of the forward pass."""
    out = {}
    D = 0.0 if dxo is None else dxo
    if pre != NONE:
        hat = normalised(xo, stats_pre)
        out["dw_pre"], out["db_pre"] = (dn * hat).sum(0), dn.sum(0)
        D = D + _through(dn * _or(w_pre, 1.0), hat, stats_pre[:, 1:], pre)
    out["dx"] = alpha * D
    if y is None:
        return out
    g, s = gate_rows(gate, span, len(D)), _or(scale, 1.0)
    hat = normalised(y, stats_post) if post != NONE else y
    u = hat * _or(w_post, 1.0) + _or(b_post, 0.0)
    if gate is not None:
        out["dgate"] = np.add.reduceat(D * s * m * u, np.arange(0, len(D), span), axis=0)
    out["dscale"] = (D * g * m * u).sum(0)
    du = D * s * g * m
    if post != NONE:
        out["dw_post"], out["db_post"] = (du * hat).sum(0), du.sum(0)
        du = _through(du * _or(w_post, 1.0), hat, stats_post[:, 1:], post)
    out["dy"] = du
    return out
