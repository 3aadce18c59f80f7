"""Float64 oracle of the feed-forward block operators: 8-bit activation
checkpoints, layer norm, activations and the linear layer's weight gradient,
each from its formula with numpy."""
from __future__ import annotations

import math

import numpy as np

GROUP = 32


def _groups(x):
    """[rows][groups][32], zeros behind the last column."""
    rows, cols = x.shape
    g = -(-cols // GROUP)
    out = np.zeros((rows, g * GROUP), np.float64)
    out[:, :cols] = x
    return out.reshape(rows, g, GROUP)


def encode(x):
    """(codes int8 [rows][pitch], exponent bytes uint8 [rows][pitch / 32]) of x.

    The step of a group with largest magnitude m in [2^p, 2^(p+1)) is 2^(p-6),
    or 2^(p-5) where m would round to 128 steps; it is at least 2^-126 and at
    most 2^121."""
    g = _groups(np.asarray(x, np.float64))
    rows, n = g.shape[:2]
    top = np.abs(g).max(2)
    bad = ~np.isfinite(top)
    safe = np.where(bad, 1.0, top)
    p = np.frexp(safe)[1] - 1
    p = np.where(safe >= 127.5 * np.exp2(p - 6.0), p + 1, p)
    p = np.clip(np.where(safe == 0, -120, p), -120, 127)
    with np.errstate(invalid="ignore"):
        q = np.clip(np.rint(g / np.exp2(p - 6.0)[..., None]), -127, 127)
    q = np.where(bad[..., None], 0, q)
    e = np.where(bad, 255, p + 127)
    return q.reshape(rows, n * GROUP).astype(np.int8), e.astype(np.uint8)


def decode(q, e, cols):
    """What the codes stand for, float64 [rows][cols]."""
    rows, n = e.shape
    step = np.where(e == 255, math.nan, np.exp2(e.astype(np.float64) - 133))
    v = q.reshape(rows, n, GROUP).astype(np.float64) * step[..., None]
    return v.reshape(rows, -1)[:, :cols]


def held(x):
    """What the checkpoint of x stands for."""
    return decode(*encode(x), x.shape[1])


def pack_bytes(q, e):
    """The checkpoint's buffer: codes, then the exponents from the next multiple
    of 256 bytes (uint8)."""
    n, m = q.size, e.size
    buf = np.zeros(-(-n // 256) * 256 + -(-m // 256) * 256, np.uint8)
    buf[:n] = q.view(np.uint8).ravel()
    at = -(-n // 256) * 256
    buf[at:at + m] = e.ravel()
    return buf


def unpack_bytes(buf, rows, cols):
    """(codes, exponents) of a checkpoint's buffer."""
    g = -(-cols // GROUP)
    n = rows * g * GROUP
    at = -(-n // 256) * 256
    return (buf[:n].view(np.int8).reshape(rows, g * GROUP),
            buf[at:at + rows * g].reshape(rows, g))


def layer_norm(t, gamma, beta, eps):
    """(y, xh, mean, rstd) of the rows of t."""
    mean = t.mean(1)
    d = t - mean[:, None]
    rstd = 1 / np.sqrt((d * d).mean(1) + eps)
    xh = d * rstd[:, None]
    return xh * gamma + beta, xh, mean, rstd


def layer_norm_backward(dy, xh, rstd, gamma, dres=None):
    """(dx, dgamma, dbeta)."""
    g = dy * gamma
    dx = rstd[:, None] * (g - g.mean(1, keepdims=True)
                          - xh * (g * xh).mean(1, keepdims=True))
    if dres is not None:
        dx = dx + dres
    return dx, (dy * xh).sum(0), dy.sum(0)


def activation(u, kind):
    """(f(u), f'(u)); kind: relu, gelu, gelu_tanh, silu."""
    if kind == "relu":
        return np.maximum(u, 0), (u > 0).astype(np.float64)
    if kind == "silu":
        s = 1 / (1 + np.exp(-u))
        return u * s, s + u * s * (1 - s)
    if kind == "gelu":
        cdf = 0.5 * np.vectorize(math.erfc, otypes=[np.float64])(-u / math.sqrt(2))
        return u * cdf, cdf + u * np.exp(-u * u / 2) / math.sqrt(2 * math.pi)
    # 0.5 (1 + tanh(z)) as 1 / (1 + exp(-2 z)): keeps its digits in the tail
    k = math.sqrt(2 / math.pi)
    with np.errstate(over="ignore"):
        s = 1 / (1 + np.exp(-2 * k * (u + 0.044715 * u ** 3)))
    return u * s, s + u * s * (1 - s) * 2 * k * (1 + 3 * 0.044715 * u * u)


def linear_wgrad(dy, q, scale=None, shift=None):
    """(dw, db) of a linear layer with input scale * q + shift."""
    x = q if scale is None else q * scale
    if shift is not None:
        x = x + shift
    return dy.T @ x, dy.sum(0)
