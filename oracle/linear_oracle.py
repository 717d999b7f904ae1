"""Plain CPU statements, in 64 bits, of what a linear layer does around the sparse product: bias, activation and
residual, their gradient, and the 8-bit activation checkpoint.  numpy and the standard library only; independent of the
CUDA library."""
from __future__ import annotations

import math

import numpy as np

NONE, RELU, GELU, GELU_TANH, SILU = range(5)
ACTS = (NONE, RELU, GELU, GELU_TANH, SILU)

_erfc = np.vectorize(math.erfc, otypes=[np.float64])
C_TANH = math.sqrt(2.0 / math.pi)


def _sigmoid(x):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-x))


def act(z, kind):
    z = np.asarray(z, dtype=np.float64)
    if kind == RELU:
        return np.where(np.isnan(z), z, np.maximum(z, 0.0))
    if kind == GELU:
        return z * 0.5 * _erfc(-z / math.sqrt(2.0))
    if kind == GELU_TANH:
        return 0.5 * z * (1.0 + np.tanh(C_TANH * (z + 0.044715 * z ** 3)))
    if kind == SILU:
        return z * _sigmoid(z)
    return z


def slope(z, kind):
    """act'(z); 0 for RELU at 0."""
    z = np.asarray(z, dtype=np.float64)
    if kind == RELU:
        return np.where(np.isnan(z), z, (z > 0).astype(np.float64))
    if kind == GELU:
        return 0.5 * _erfc(-z / math.sqrt(2.0)) + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if kind == GELU_TANH:
        t = np.tanh(C_TANH * (z + 0.044715 * z ** 3))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * C_TANH * (1.0 + 3.0 * 0.044715 * z * z)
    if kind == SILU:
        s = _sigmoid(z)
        return s * (1.0 + z * (1.0 - s))
    return np.ones_like(z)


def linear(X, Wm, bias, kind, R):
    """(Y, Z) of Y = act(X Wm^T + bias) + R for a masked I x J matrix Wm."""
    z = np.asarray(X, np.float64) @ np.asarray(Wm, np.float64).T
    if bias is not None:
        z = z + np.asarray(bias, np.float64)
    y = act(z, kind)
    return (y if R is None else y + np.asarray(R, np.float64)), z


def act_bwd(dY, z, kind):
    """(dZ, dbias)."""
    dz = np.asarray(dY, np.float64) * slope(z, kind)
    return dz, dz.sum(axis=0)


LARGEST = 127.0 * 2.0 ** 121          # the next scale, 2^122, would round a larger magnitude to 64 steps: 2^128, infinity in bf16


def pack(x):
    """Checkpoint of a T x C matrix: signed bytes q, scale bytes s (q is zero where s = 255)."""
    x = np.asarray(x, np.float64)
    b = x.reshape(x.shape[0], -1, 32)
    q = np.zeros(b.shape, np.int8)
    s = np.zeros(b.shape[:2], np.uint8)
    for t in range(b.shape[0]):
        for g in range(b.shape[1]):
            v = b[t, g]
            m = np.max(np.abs(v))
            if not m <= LARGEST:                                # NaN and infinity included
                s[t, g] = 255
                continue
            e = -126
            while m > 127.0 * 2.0 ** e:
                e += 1
            s[t, g] = e + 127
            q[t, g] = np.rint(v / 2.0 ** e).astype(np.int8)     # rint: ties to even
    return q.reshape(x.shape), s


def unpack(q, s):
    q = np.asarray(q, np.float64)
    scale = np.where(s == 255, np.nan, np.where(s == 0, 0.0, np.exp2(s.astype(np.float64) - 127.0)))
    return (q.reshape(q.shape[0], -1, 32) * scale[..., None]).reshape(q.shape)


def wgrad(dY, x):
    return np.asarray(dY, np.float64).T @ np.asarray(x, np.float64)
