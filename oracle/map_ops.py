"""Float64 oracle of group norm with an activation, dropout's generator and the
gated feed-forward block, each from its formula with numpy."""
from __future__ import annotations

import numpy as np

from .block import activation


def _act(t, kind):
    return (t, np.ones_like(t)) if kind == "none" else activation(t, kind)


def _by_group(x, batch, groups):
    return x.reshape(batch, x.shape[0] // batch, groups, x.shape[1] // groups)


def spread(s, pixels, cols):
    """[batch][groups] over the rows and columns of the map."""
    per = np.repeat(s, cols // s.shape[1], 1)
    return np.repeat(per[:, None], pixels, 1).reshape(-1, cols)


def group_norm(x, batch, groups, gamma, beta, eps, kind):
    """(y, t, xh, mean, rstd): t before the activation."""
    g = _by_group(x, batch, groups)
    mean = g.mean((1, 3))
    d = g - mean[:, None, :, None]
    rstd = 1 / np.sqrt((d * d).mean((1, 3)) + eps)
    xh = (d * rstd[:, None, :, None]).reshape(x.shape)
    t = xh * gamma + beta
    return _act(t, kind)[0], t, xh, mean, rstd


def group_norm_backward(dy, xh, rstd, batch, groups, gamma, beta, kind):
    """(dx, dgamma, dbeta)."""
    e = dy * _act(xh * gamma + beta, kind)[1]
    q, h = _by_group(e * gamma, batch, groups), _by_group(xh, batch, groups)
    m1, m2 = q.mean((1, 3), keepdims=True), (q * h).mean((1, 3), keepdims=True)
    dx = rstd[:, None, :, None] * (q - m1 - h * m2)
    return dx.reshape(dy.shape), (e * xh).sum(0), e.sum(0)


def philox4x32(counter, key, rounds=10):
    """The four output words (uint64 arrays below 2^32) of Philox4x32 (Salmon, Moraes,
    Dror and Shaw, SC 2011)."""
    m = np.uint64(0xFFFFFFFF)
    c = [np.asarray(w, np.uint64) for w in counter]
    k0, k1 = int(key[0]), int(key[1])
    for _ in range(rounds):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        s = np.uint64(32)
        c = [(q >> s) ^ c[1] ^ np.uint64(k0), q & m, (p >> s) ^ c[3] ^ np.uint64(k1), p & m]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c


def dropout_bits(seed, offset, rows, cols, site=0, first_row=0):
    """The 16 random bits of each element."""
    seed, offset = seed % 2 ** 64, offset % 2 ** 64
    per = -(-cols // 8)
    g = (np.uint64(first_row) + np.arange(rows, dtype=np.uint64)[:, None]) * np.uint64(per) \
        + np.arange(per, dtype=np.uint64)
    low, s = np.uint64(0xFFFFFFFF), np.uint64(32)
    full = lambda v: np.full(g.shape, v, np.uint64)
    words = philox4x32([g & low, (g >> s) | np.uint64(site << 16), full(offset % 2 ** 32),
                        full(offset >> 32)], (seed % 2 ** 32, seed >> 32))
    out = np.empty((rows, per, 8), np.int64)
    for i, w in enumerate(words):
        out[..., 2 * i] = w & np.uint64(0xFFFF)
        out[..., 2 * i + 1] = w >> np.uint64(16)
    return out.reshape(rows, per * 8)[:, :cols]


def dropout(x, p, bits, residual=None):
    least = int(np.rint(65536 * p))
    scale = 65536 / (65536 - least) if least < 65536 else 0.0
    y = np.where(bits >= least, x, 0.0) * scale
    return y if residual is None else y + residual


def gated(x, w1, b1, kind):
    """(u, v, f(u) v)."""
    uv = x @ w1.T + b1
    u, v = uv[:, :w1.shape[0] // 2], uv[:, w1.shape[0] // 2:]
    return u, v, activation(u, kind)[0] * v


def gated_backward(da, u, v, kind):
    """(du, dv)."""
    f, df = activation(u, kind)
    return da * df * v, da * f
