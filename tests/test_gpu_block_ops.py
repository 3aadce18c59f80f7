"""The feed-forward block operators on the GPU against the float64 oracle: 8-bit
activation checkpoints, layer norm, activations, and the weight gradient that
reads a checkpoint -- from one row and one column on, odd and ragged widths,
slices with odd strides, no rows at all, values that are not finite, and
offsets past 32 bits.

Tolerances, with u = 2^-24 (float32 rounding) and D additions on the longest
path of a sum: a sum is off by at most D u times the sum of magnitudes. Layer
norm: 8 columns of up to 4 vectors in a thread, 4 + 2 steps across a wave, up
to 8 waves, so D <= 46, and a few roundings more: 4e-6 (64 u). Sums over rows:
at most 160 in a row, 1e-5. A bfloat16 result adds half an ulp, 2^-9 of the
value, taken as 2^-8 where the value itself is uncertain by the float32 error.
Codes of a given input are exact."""
import math

import numpy as np
import pytest
import torch

from oracle import block as OB
from paper_2401_11471_amd import lrcnn as L

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
TYPES = pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
KINDS = {"relu": L.ACT_RELU, "gelu": L.ACT_GELU, "gelu_tanh": L.ACT_GELU_TANH, "silu": L.ACT_SILU}
SHAPES = [(1, 1), (1, 7), (2, 8), (3, 31), (5, 32), (4, 33), (65, 64), (1, 509), (130, 512),
          (9, 513), (33, 1000), (2, 2048), (700, 2049), (3, 4097), (6, 8200), (2, 16384)]
SIZES = pytest.mark.parametrize("rows,cols", SHAPES)


def tell(*a):
    print(*a, flush=True)


def matrix(a, dtype, pad=0, at=0):
    """a on the GPU; pad > 0: a slice of a wider matrix from column `at`, NaN
    around it."""
    t = torch.from_numpy(np.asarray(a, np.float32)).to("cuda", dtype)
    if not pad:
        return t.contiguous()
    rows, cols = t.shape
    wide = torch.full((rows, cols + pad), float("nan"), device="cuda", dtype=dtype)
    s = wide[:, at:at + cols]
    s.copy_(t)
    return s


def vec(a):
    return torch.from_numpy(np.asarray(a, np.float32)).cuda()


def np64(t):
    return t.double().cpu().numpy()


def buf(n):
    return torch.full((max(int(n), 16),), 0xA5, device="cuda", dtype=torch.uint8)


def ckpt(rows, cols):
    return buf(L.lrcnn_act8_bytes(rows, cols))


def checkpoint_of(x):
    """A checkpoint on the GPU, made by the oracle, and what it stands for."""
    q, e = OB.encode(x)
    b = OB.pack_bytes(q, e)
    return torch.from_numpy(b).cuda(), OB.decode(q, e, x.shape[1])


def rounded(x, dtype):
    return np64(matrix(x, dtype)) if x.size else x


def out_tol(ref, dtype):
    return np.abs(ref) * (2.0 ** -8 if dtype == BF16 else 0) + 1e-37


def close(got, ref, tol):
    got = np64(got)
    assert got.shape == ref.shape
    assert np.isfinite(got).all()
    over = np.abs(got - ref) - tol
    assert (over <= 0).all(), f"off by {np.abs(got - ref).max():.3g}, {over.max():.3g} over"


def features(rng, rows, cols):
    x = rng.standard_normal((rows, cols)) * np.exp(0.5 * rng.standard_normal(cols))
    return x + 0.5 * rng.standard_normal(cols)


# ------------------------------------------------------------- checkpoints
@TYPES
@SIZES
def test_pack_is_the_oracles_bytes(rows, cols, dtype):
    tell("pack", rows, cols, dtype)
    rng = np.random.default_rng(rows + cols)
    x = features(rng, rows, cols) * np.exp(rng.uniform(-20, 20, (rows, 1)))
    if rows > 2:
        x[1] = 0
    for pad, at in [(0, 0), (3, 1), (5, 2)]:
        t = matrix(x, dtype, pad, at)
        q, e = OB.encode(np64(t))
        c = ckpt(rows, cols)
        L.lrcnn_act8_pack(t, c)
        got = c.cpu().numpy()
        gq, ge = OB.unpack_bytes(got, rows, cols)
        assert np.array_equal(ge, e) and np.array_equal(gq, q)
        for od in (F32, BF16):
            y = matrix(np.zeros((rows, cols)), od, pad, at)
            L.lrcnn_act8_unpack(c, y)
            assert np.array_equal(np64(y), OB.decode(q, e, cols))
    if pad:  # nothing beside the slice was written
        assert torch.isnan(y._base[:, :at]).all() and torch.isnan(y._base[:, at + cols:]).all()


@TYPES
def test_pack_edges(dtype):
    lowest = torch.finfo(dtype).min
    x = np.zeros((12, 96))
    x[0, 5], x[1, 40], x[2, 95] = math.nan, math.inf, -math.inf
    x[3, :] = lowest
    x[4, ::7] = lowest
    x[5, 0] = 2.0 ** -126
    x[6, 3] = 2.0 ** -130
    x[7, :3] = [2.0 - 2.0 ** -7, 2.5 / 64, -3.5 / 64]
    x[8, :4] = [1.0, 2.5 / 64, 3.5 / 64, -2.5 / 64]
    x[9, :] = -0.0
    x[10, 64:] = 3e38
    t = torch.from_numpy(x).to("cuda", dtype)
    c = ckpt(12, 96)
    L.lrcnn_act8_pack(t, c)
    q, e = OB.encode(np64(t))
    gq, ge = OB.unpack_bytes(c.cpu().numpy(), 12, 96)
    assert np.array_equal(ge, e) and np.array_equal(gq, q)
    y = torch.empty(12, 96, device="cuda", dtype=dtype)
    L.lrcnn_act8_unpack(c, y)
    assert np.array_equal(np64(y), OB.decode(q, e, 96), equal_nan=True)
    assert torch.isnan(y[0, :32]).all() and torch.isfinite(y[0, 32:]).all()
    assert (y[3] == -127 * 2.0 ** 121).all()


def test_pack_past_32_bits():
    """More than 2^32 bytes of codes, in joined rows and in rows of ragged width."""
    for rows, cols in [(1 << 20, 4128), (1 << 20, 4100)]:
        tell("pack", rows, cols)
        x = torch.zeros(rows, cols, device="cuda", dtype=BF16)
        x[-3:] = torch.randn(3, cols, device="cuda")
        x[rows // 2] = 1.0
        c = torch.empty(L.lrcnn_act8_bytes(rows, cols), device="cuda", dtype=torch.uint8)
        L.lrcnn_act8_pack(x, c)
        y = torch.full_like(x, float("nan"))
        L.lrcnn_act8_unpack(c, y)
        assert np.array_equal(np64(y[-3:]), OB.held(np64(x[-3:])))
        assert (y[rows // 2] == 1).all()
        assert int(torch.count_nonzero(y)) == cols + int(torch.count_nonzero(y[-3:]))
        del x, y, c
        torch.cuda.empty_cache()


# -------------------------------------------------------------- layer norm
def held_ok(c, xh, tol):
    """A checkpoint of computed values xh: its values within half a step of
    them, its steps the oracle's but where the largest value is within the
    tolerance of a boundary."""
    rows, cols = xh.shape
    q, e = OB.unpack_bytes(c.cpu().numpy(), rows, cols)
    _, want = OB.encode(xh)
    step = np.exp2(e.astype(float) - 133)
    got = OB.decode(q, e, cols)
    half = np.repeat(step / 2, 32, axis=1)[:, :cols]
    assert (np.abs(got - xh) <= half + tol).all()
    lo = np.minimum(e, want).astype(float)
    assert (np.maximum(e, want) - lo <= 1).all()
    top, slack = (np.abs(OB._groups(t)).max(2) for t in (xh, np.broadcast_to(tol, xh.shape)))
    near = np.abs(top - 127.5 * np.exp2(lo - 133)) <= slack
    assert (near | (e == want)).all()
    if cols % 32:
        assert (q[:, cols:] == 0).all()


@TYPES
@SIZES
@pytest.mark.parametrize("full", [True, False], ids=["all", "plain"])
def test_layer_norm_forward(rows, cols, dtype, full):
    tell("ln_fwd", rows, cols, dtype, full)
    rng = np.random.default_rng(7 * rows + cols)
    pad, at = (3, 1) if full else (0, 0)
    x = matrix(features(rng, rows, cols), dtype, pad, at)
    ga, be = 1 + 0.3 * rng.standard_normal(cols), rng.standard_normal(cols)
    ga, be = np64(vec(ga)), np64(vec(be))
    y = matrix(np.zeros((rows, cols)), dtype, pad, at)
    t = np64(x)
    if full:
        res = matrix(features(rng, rows, cols), dtype, 2, 2)
        total = matrix(np.zeros((rows, cols)), dtype, 1, 0)
        mean, rstd, c = vec(np.zeros(rows)), vec(np.zeros(rows)), ckpt(rows, cols)
        L.lrcnn_layer_norm_forward(x, vec(ga), vec(be), 1e-5, y, residual=res, total=total,
                                   mean=mean, rstd=rstd, ckpt=c)
        t = np64((x.float() + res.float()).to(dtype))
        assert np.array_equal(np64(total), t)
    else:
        L.lrcnn_layer_norm_forward(x, None, None, 1e-5, y)
        ga, be = np.ones(cols), np.zeros(cols)
    ry, xh, rm, rr = OB.layer_norm(t, ga, be, 1e-5)
    # the mean is off by 64 u mean|t|, xh by that times rstd and 64 u of itself;
    # the variance by 64 u and the mean's error squared
    dm = 4e-6 * np.abs(t).mean(1)
    dxh = (dm * rr)[:, None] * (1 + np.abs(xh)) + 4e-6 * np.abs(xh)
    close(y, ry, np.abs(ga) * dxh + 4e-6 * np.abs(be) + out_tol(ry, dtype))
    if full:
        close(mean, rm, dm + 1e-37)
        close(rstd, rr, rr * (4e-6 + dm * rr))
        held_ok(c, xh, dxh)
        assert torch.isnan(y._base[:, 0]).all() and torch.isnan(y._base[:, at + cols:]).all()


@TYPES
@SIZES
@pytest.mark.parametrize("saved", [True, False], ids=["ckpt", "x"])
def test_layer_norm_backward(rows, cols, dtype, saved):
    tell("ln_bwd", rows, cols, dtype, saved)
    rng = np.random.default_rng(11 * rows + cols)
    pad, at = (3, 1) if saved else (0, 0)
    x = matrix(features(rng, rows, cols), dtype, pad, at)
    dy = matrix(rng.standard_normal((rows, cols)) * (rng.random((rows, 1)) > 0.1), dtype, pad, at)
    ga = np64(vec(1 + 0.3 * rng.standard_normal(cols)))
    _, xh, rm, rr = OB.layer_norm(np64(x), ga, 0, 1e-3)
    mean, rstd = vec(rm), vec(rr)
    dres = None
    if saved:
        c, xh = checkpoint_of(xh)
        dres = matrix(rng.standard_normal((rows, cols)), dtype, 4, 3)
        src = dict(ckpt=c, dres=dres)
    else:
        xh = (np64(x) - np64(mean)[:, None]) * np64(rstd)[:, None]
        src = dict(x=x, mean=mean)
    dx = matrix(np.zeros((rows, cols)), dtype, pad, at)
    dg, db = vec(np.full(cols, 3.0)), vec(np.full(cols, -2.0))
    ws = buf(L.lrcnn_layer_norm_workspace_bytes(rows, cols))
    d64, rs = np64(dy), np64(rstd)
    rdx, rdg, rdb = OB.layer_norm_backward(d64, xh, rs, ga, None if dres is None else np64(dres))
    g = np.abs(d64 * ga)
    # g, mean(g), xh mean(g xh): 64 u each; xh from x by 4 u of |x - mean| and
    # of the mean itself, which cancels against x
    exh = 0 if saved else 4e-7 * (np.abs(xh) + (np.abs(np64(x)) * rs[:, None]))
    m1, m2 = g.mean(1, keepdims=True), (g * np.abs(xh)).mean(1, keepdims=True)
    tol = rs[:, None] * (4e-6 * (g + m1 + np.abs(xh) * m2) + exh * m2
                         + np.abs(xh) * (g * exh).mean(1, keepdims=True))
    if dres is not None:
        tol = tol + 4e-6 * np.abs(np64(dres))
    for acc in (False, True):
        L.lrcnn_layer_norm_backward(dy, rstd, vec(ga), dx, dg, db, ws, accumulate=acc, **src)
        close(dx, rdx, tol + out_tol(rdx, dtype))
        k = 2 if acc else 1
        close(dg, k * rdg, k * (1e-5 * np.abs(d64 * xh).sum(0) + (np.abs(d64) * exh).sum(0)) + 1e-37)
        close(db, k * rdb, k * 1e-5 * np.abs(d64).sum(0) + 1e-37)
    if pad:
        assert torch.isnan(dx._base[:, 0]).all() and torch.isnan(dx._base[:, at + cols:]).all()
    # dx alone, over dy
    L.lrcnn_layer_norm_backward(dy, rstd, vec(ga), dy, **src)
    assert torch.equal(dy, dx)


def test_layer_norm_backward_against_differences():
    """dL/dx, dL/dgamma, dL/dbeta of the kernels along a direction against the
    central difference of the float64 forward pass."""
    rng = np.random.default_rng(3)
    rows, cols, h = 37, 200, 1e-5
    x, w = rng.standard_normal((2, rows, cols))
    x, w = np64(vec(x)), np64(vec(w))
    ga, be = np64(vec(1 + 0.3 * rng.standard_normal(cols))), np.zeros(cols)
    mean, rstd = vec(np.zeros(rows)), vec(np.zeros(rows))
    y, dx = torch.empty(2, rows, cols, device="cuda").unbind(0)
    dg, db = vec(be), vec(be)
    L.lrcnn_layer_norm_forward(vec(x), vec(ga), vec(be), 1e-3, y, mean=mean, rstd=rstd)
    ws = buf(L.lrcnn_layer_norm_workspace_bytes(rows, cols))
    L.lrcnn_layer_norm_backward(vec(w), rstd, vec(ga), dx, dg, db, ws, x=vec(x), mean=mean)

    def loss(x, ga, be):
        return (OB.layer_norm(x, ga, be, 1e-3)[0] * w).sum()
    for _ in range(3):
        d = rng.standard_normal((rows, cols))
        diff = (loss(x + h * d, ga, be) - loss(x - h * d, ga, be)) / (2 * h)
        assert (np64(dx) * d).sum() == pytest.approx(diff, abs=1e-5 * np.abs(np64(dx) * d).sum())
        e = rng.standard_normal(cols)
        diff = (loss(x, ga + h * e, be) - loss(x, ga - h * e, be)) / (2 * h)
        assert (np64(dg) * e).sum() == pytest.approx(diff, abs=1e-5 * np.abs(np64(dg) * e).sum())
        diff = (loss(x, ga, be + h * e) - loss(x, ga, be - h * e)) / (2 * h)
        assert (np64(db) * e).sum() == pytest.approx(diff, abs=1e-5 * np.abs(np64(db) * e).sum())


@TYPES
def test_layer_norm_of_constant_large_and_bad_rows(dtype):
    rows, cols = 6, 96
    rng = np.random.default_rng(1)
    x = rng.standard_normal((rows, cols))
    x[0] = 0
    x[1] = 4.0
    x[2] += 512          # a mean far over the spread
    x[3, 7] = math.nan
    x[4, 9] = math.inf
    t = matrix(x, dtype)
    y, c = torch.empty_like(t), ckpt(rows, cols)
    mean, rstd = vec(np.zeros(rows)), vec(np.zeros(rows))
    L.lrcnn_layer_norm_forward(t, None, None, 1e-5, y, mean=mean, rstd=rstd, ckpt=c)
    assert (y[:2] == 0).all() and np.allclose(np64(rstd[:2]), 1e-5 ** -0.5, rtol=1e-6)
    ry, _, _, rr = OB.layer_norm(np64(t), np.ones(cols), 0, 1e-5)
    close(y[2:3], ry[2:3], 4e-6 * 512 * rr[2] * 3 + out_tol(ry[2:3], dtype))
    assert torch.isnan(y[3:5]).all()
    close(y[5:], ry[5:], 2e-5 + out_tol(ry[5:], dtype))
    h = torch.empty_like(t)
    L.lrcnn_act8_unpack(c, h)
    assert (h[:2] == 0).all() and torch.isnan(h[3:5]).all() and torch.isfinite(h[5]).all()


def test_layer_norm_past_32_bits():
    rows, cols = 300000, 8192
    tell("layer norm", rows, cols)
    x = torch.zeros(rows, cols, device="cuda", dtype=BF16)
    x[-2:] = torch.randn(2, cols, device="cuda")
    y = torch.full_like(x, float("nan"))
    c = torch.empty(L.lrcnn_act8_bytes(rows, cols), device="cuda", dtype=torch.uint8)
    mean, rstd = torch.empty(2, rows, device="cuda").unbind(0)
    L.lrcnn_layer_norm_forward(x, None, None, 1e-5, y, mean=mean, rstd=rstd, ckpt=c)
    ry, _, _, rr = OB.layer_norm(np64(x[-2:]), np.ones(cols), 0, 1e-5)
    close(y[-2:], ry, 4e-5 + out_tol(ry, BF16))
    assert int(torch.count_nonzero(y[:-2])) == 0
    # backward: only the last two rows carry a gradient
    dx = torch.full_like(x, float("nan"))
    dg, db = torch.empty(2, cols, device="cuda").unbind(0)
    ws = buf(L.lrcnn_layer_norm_workspace_bytes(rows, cols))
    held = torch.empty_like(x)
    L.lrcnn_act8_unpack(c, held)
    L.lrcnn_layer_norm_backward(x, rstd, None, dx, dg, db, ws, ckpt=c)
    rdx, rdg, rdb = OB.layer_norm_backward(np64(x[-2:]), np64(held[-2:]), np64(rstd[-2:]),
                                           np.ones(cols))
    close(dx[-2:], rdx, 4e-5 + out_tol(rdx, BF16))
    close(dg, rdg, 1e-5 * (1 + np.abs(rdg)))
    close(db, rdb, 1e-5 * (1 + np.abs(rdb)))
    assert int(torch.count_nonzero(dx[:-2])) == 0


# ------------------------------------------------------------- activations
def f_tol(u, f):
    """f: the fit's 4.4e-7 and the exponent's rounding, u^2 / 2 or |u| times u."""
    return np.abs(f) * (1e-6 + 2e-7 * u * u) + 1e-37


@TYPES
@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("gated", [False, True], ids=["one", "gated"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 31), (4, 32), (7, 100), (300, 64), (2, 4097),
                                       (65, 2048)])
def test_activation(rows, cols, kind, gated, dtype):
    tell("activation", rows, cols, kind, gated, dtype)
    rng = np.random.default_rng(rows + 3 * cols)
    uv = matrix(3 * rng.standard_normal((rows, 2 * cols)), dtype)
    u = uv[:, :cols] if gated else uv[:, :cols].contiguous()
    v = uv[:, cols:] if gated else None
    a, ku, ka = torch.empty(rows, cols, device="cuda", dtype=dtype), ckpt(rows, cols), ckpt(rows, cols)
    kv = ckpt(rows, cols) if gated else None
    L.lrcnn_activation_forward(KINDS[kind], u, a, v=v, ckpt_u=ku, ckpt_v=kv, ckpt_a=ka)
    u64 = np64(u)
    f, _ = OB.activation(u64, kind)
    w = np64(v) if gated else 1.0
    tol = f_tol(u64, f) * np.abs(w)
    close(a, f * w, tol + out_tol(f * w, dtype))
    held_ok(ka, f * w, tol + 1e-7 * np.abs(f * w))
    for k, x in ((ku, u), (kv, v)):
        if k is not None:
            q, e = OB.unpack_bytes(k.cpu().numpy(), rows, cols)
            rq, re = OB.encode(np64(x))
            assert np.array_equal(q, rq) and np.array_equal(e, re)
    da = matrix(rng.standard_normal((rows, cols)), dtype)
    d64 = np64(da)
    for saved in (False, True):
        duv = torch.full((rows, 2 * cols), float("nan"), device="cuda", dtype=dtype)
        du, dv = duv[:, :cols], duv[:, cols:] if gated else None
        src = dict(ckpt_u=ku, ckpt_v=kv) if saved else dict(u=u, v=v)
        u64 = OB.held(np64(u)) if saved else np64(u)
        w = (OB.held(np64(v)) if saved else np64(v)) if gated else np.ones((1, 1))
        f, df = OB.activation(u64, kind)
        k2 = ckpt(rows, cols)
        L.lrcnn_activation_backward(KINDS[kind], da, du, dv=dv, ckpt_a=k2, **src)
        close(du, d64 * df * w, 3e-6 * np.abs(d64 * w) + out_tol(d64 * df * w, dtype))
        if gated:
            close(dv, d64 * f, f_tol(u64, f) * np.abs(d64) + 1e-7 * np.abs(d64 * f)
                  + out_tol(d64 * f, dtype))
        else:
            assert torch.isnan(duv[:, cols:]).all()
        held_ok(k2, f * w, f_tol(u64, f) * np.abs(w) + 1e-7 * np.abs(f * w))


@pytest.mark.parametrize("kind", list(KINDS))
def test_activation_limits(kind):
    u = torch.tensor([[math.inf, -math.inf, 1e30, -1e30, 150.0, -150.0, 0.0, -0.0, math.nan,
                       88.0, -88.0, -14.5, 14.5]], device="cuda")
    a, du, one = torch.empty_like(u), torch.empty_like(u), torch.ones_like(u)
    L.lrcnn_activation_forward(KINDS[kind], u, a)
    L.lrcnn_activation_backward(KINDS[kind], one, du, u=u)
    assert torch.isnan(a[0, 8]) and torch.isnan(du[0, 8])
    a, du = np64(a)[0], np64(du)[0]
    assert a[0] == math.inf and a[2] == np.float32(1e30) and a[4] == 150
    assert np.abs(a[[1, 3, 5, 6, 7]]).max() < 1e-30
    half = 0.0 if kind == "relu" else 0.5
    assert np.allclose(du[[0, 1, 2, 3, 4, 5, 6, 7, 9, 10]],
                       [1, 0, 1, 0, 1, 0, half, half, 1, 0], atol=1e-6)
    f, _ = OB.activation(np.array([-14.5, 14.5]), kind)
    assert np.allclose(a[11:], f, rtol=5e-5, atol=1e-37)


@pytest.mark.parametrize("kind", list(KINDS))
def test_activation_gradient_against_differences(kind):
    rng = np.random.default_rng(9)
    u, v, w = (np64(vec(t)) for t in rng.standard_normal((3, 20, 50)))
    du, dv = torch.empty(2, 20, 50, device="cuda").unbind(0)
    L.lrcnn_activation_backward(KINDS[kind], vec(w), du, u=vec(u), v=vec(v), dv=dv)
    h = 1e-6
    for x, g, at in ((u, du, 0), (v, dv, 1)):
        d = rng.standard_normal(x.shape)

        def loss(t):
            p, q = (t, v) if at == 0 else (u, t)
            return (OB.activation(p, kind)[0] * q * w).sum()
        diff = (loss(x + h * d) - loss(x - h * d)) / (2 * h)
        assert (np64(g) * d).sum() == pytest.approx(diff, abs=1e-5 * np.abs(np64(g) * d).sum())


# --------------------------------------------------------- weight gradient
@TYPES
@pytest.mark.parametrize("rows,n_in,n_out", [
    (0, 5, 3), (1, 1, 1), (1, 32, 8), (3, 33, 7), (31, 31, 129), (32, 128, 128), (33, 100, 130),
    (300, 509, 1000), (1000, 130, 64), (5000, 64, 10), (4097, 257, 65), (600, 1024, 512),
    (2500, 300, 515)])
@pytest.mark.parametrize("affine", [False, True], ids=["plain", "affine"])
def test_linear_wgrad(rows, n_in, n_out, dtype, affine):
    tell("wgrad", rows, n_in, n_out, dtype, affine)
    rng = np.random.default_rng(rows + n_in + n_out)
    x = features(rng, rows, n_in)
    if rows:
        c, q = checkpoint_of(x)
        dy = matrix(rng.standard_normal((rows, n_out)) * (rng.random((rows, 1)) > 0.1), dtype,
                    3 if affine else 0, 1 if affine else 0)
    else:
        c, q = buf(16), x
        dy = torch.empty(0, n_out, device="cuda", dtype=dtype)
    sc = sh = None
    if affine:
        sc, sh = np64(vec(1 + 0.3 * rng.standard_normal(n_in))), np64(vec(rng.standard_normal(n_in)))
    dw = torch.full((n_out, n_in), 2.0, device="cuda")
    db = torch.full((n_out,), -1.0, device="cuda")
    ws = buf(L.lrcnn_linear_wgrad_workspace_bytes(rows, n_in, n_out,
                                                  L.BF16 if dtype == BF16 else L.F32))
    d64 = np64(dy)
    rw, rb = OB.linear_wgrad(d64, q, sc, sh)
    tw, tb = OB.linear_wgrad(np.abs(d64), np.abs(q), None if sc is None else np.abs(sc),
                             None if sh is None else np.abs(sh))
    gv = dict(scale=None if sc is None else vec(sc), shift=None if sh is None else vec(sh))
    L.lrcnn_linear_wgrad(dy, c, dw, ws, db=db, **gv)
    close(dw, rw, 1e-5 * tw + 1e-37)
    close(db, rb, 1e-5 * tb + 1e-37)
    one = dw.clone()
    L.lrcnn_linear_wgrad(dy, c, dw, ws, db=db, accumulate=True, **gv)
    close(dw, 2 * rw, 3e-5 * tw + 1e-37)
    close(db, 2 * rb, 3e-5 * tb + 1e-37)
    L.lrcnn_linear_wgrad(dy, c, dw, ws, **gv)
    assert torch.equal(dw, one)  # again, without db: the same bits


@TYPES
def test_linear_wgrad_of_values_that_are_not_finite(dtype):
    """A group that stands for NaN reaches its 32 columns of dw and no other; a
    row of dy with an infinity its own rows."""
    rng = np.random.default_rng(2)
    rows, n_in, n_out = 100, 200, 70
    x = rng.standard_normal((rows, n_in))
    x[17, 40] = math.nan
    c, q = checkpoint_of(x)
    dy = matrix(rng.standard_normal((rows, n_out)), dtype)
    dw, ws = torch.empty(n_out, n_in, device="cuda"), buf(1 << 20)
    L.lrcnn_linear_wgrad(dy, c, dw, ws)
    bad = torch.isnan(dw)
    assert bad[:, 32:64].all() and not bad[:, :32].any() and not bad[:, 64:].any()
    dy[30, 3] = math.inf
    c, q = checkpoint_of(rng.standard_normal((rows, n_in)) + 10)
    L.lrcnn_linear_wgrad(dy, c, dw, ws)
    assert not torch.isfinite(dw[3]).any()
    assert torch.isfinite(dw[:3]).all() and torch.isfinite(dw[4:]).all()


def test_linear_wgrad_float32_keeps_its_digits():
    """dy of 24 significant bits whose leading 8 cancel between rows: a product
    in bfloat16 or two pieces would lose the result."""
    n = 64
    dy = np.zeros((2, n))
    dy[0] = 1.0 + np.arange(1, n + 1) * 2.0 ** -23
    dy[1] = -1.0
    c, q = checkpoint_of(np.ones((2, 32)))
    dw = torch.empty(n, 32, device="cuda")
    L.lrcnn_linear_wgrad(matrix(dy, F32), c, dw)
    assert np.array_equal(np64(dw), np.repeat((np.arange(1, n + 1) * 2.0 ** -23)[:, None], 32, 1))


def test_linear_wgrad_past_32_bits():
    rows, n_in, n_out = (1 << 21) + 5, 2080, 16
    tell("wgrad", rows, n_in, n_out)
    x = torch.zeros(rows, n_in, device="cuda", dtype=BF16)
    x[-3:] = torch.randn(3, n_in, device="cuda")
    c = torch.empty(L.lrcnn_act8_bytes(rows, n_in), device="cuda", dtype=torch.uint8)
    L.lrcnn_act8_pack(x, c)
    q = OB.held(np64(x[-3:]))
    del x
    dy = torch.randn(rows, n_out, device="cuda").bfloat16()
    dw = torch.empty(n_out, n_in, device="cuda")
    ws = buf(L.lrcnn_linear_wgrad_workspace_bytes(rows, n_in, n_out, L.BF16))
    L.lrcnn_linear_wgrad(dy, c, dw, ws)
    d = np64(dy[-3:])
    close(dw, d.T @ q, 1e-5 * np.abs(d).T @ np.abs(q) + 1e-37)


# ------------------------------------------------------- streams and graphs
def test_runs_on_the_callers_stream_and_in_a_graph():
    """All operators of a block's step on another stream, then captured and
    replayed on new inputs between eager work: the same bits as eager calls."""
    rows, cols, hid = 70, 96, 200
    g = torch.Generator(device="cuda").manual_seed(4)

    def n(*s):
        return torch.randn(*s, generator=g, device="cuda")
    x, res, dh, dy, u, dr = (n(rows, c).bfloat16() for c in (cols, cols, hid, cols, hid, cols))
    ga, be = n(cols), n(cols)
    out = {}

    def e(name, *s, dtype=BF16):
        out[name] = torch.full(s, 7, device="cuda", dtype=dtype)
        return out[name]
    y, tot, dx = (e(k, rows, cols) for k in ("y", "tot", "dx"))
    a, du = e("a", rows, hid), e("du", rows, hid)
    mean, rstd = e("mean", rows, dtype=F32), e("rstd", rows, dtype=F32)
    dg, db = e("dg", cols, dtype=F32), e("db", cols, dtype=F32)
    dw, dbw = e("dw", hid, cols, dtype=F32), e("dbw", hid, dtype=F32)
    kx, ku, ka = ckpt(rows, cols), ckpt(rows, hid), ckpt(rows, hid)
    ws1 = buf(L.lrcnn_layer_norm_workspace_bytes(rows, cols))
    ws2 = buf(L.lrcnn_linear_wgrad_workspace_bytes(rows, cols, hid, L.BF16))

    def step():
        L.lrcnn_layer_norm_forward(x, ga, be, 1e-5, y, residual=res, total=tot, mean=mean,
                                   rstd=rstd, ckpt=kx)
        L.lrcnn_activation_forward(L.ACT_GELU, u, a, ckpt_u=ku)
        L.lrcnn_activation_backward(L.ACT_GELU, dh, du, ckpt_u=ku, ckpt_a=ka)
        L.lrcnn_linear_wgrad(du, kx, dw, ws2, db=dbw, scale=ga, shift=be)
        L.lrcnn_layer_norm_backward(dy, rstd, ga, dx, dg, db, ws1, ckpt=kx, dres=dr)

    def snapshot():
        torch.cuda.synchronize()
        return {k: v.clone() for k, v in out.items()}
    side = torch.cuda.Stream()
    step()
    want = snapshot()
    for v in out.values():
        v.fill_(7)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    got = snapshot()
    assert all(torch.equal(got[k], want[k]) for k in want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        x.copy_(n(rows, cols))
        u.copy_(n(rows, hid))
        step()
        want = snapshot()
        for v in out.values():
            v.fill_(7)
        graph.replay()
        got = snapshot()
        assert all(torch.equal(got[k], want[k]) for k in want)


# ----------------------------------------- the sizes at which kernels change
NARROW = [(70, 65), (41, 100), (130, 128), (19, 129), (66, 200), (257, 256), (12, 257), (33, 640),
          (5, 1024), (18, 1025), (3, 4096), (2, 8192), (300000, 17), (100001, 33)]


@TYPES
@pytest.mark.parametrize("rows,cols", NARROW)
@pytest.mark.parametrize("full", [True, False], ids=["all", "plain"])
def test_layer_norm_forward_widths(rows, cols, dtype, full):
    """Widths on both sides of those at which a row takes more threads, and rows
    enough that a block takes several."""
    test_layer_norm_forward(rows, cols, dtype, full)


@TYPES
@pytest.mark.parametrize("rows,cols", NARROW)
@pytest.mark.parametrize("saved", [True, False], ids=["ckpt", "x"])
def test_layer_norm_backward_widths(rows, cols, dtype, saved):
    test_layer_norm_backward(rows, cols, dtype, saved)


@TYPES
@pytest.mark.parametrize("rows,n_in,n_out", [
    (1, 4096, 4096), (33, 2500, 5000), (64, 2048, 8192), (65, 4096, 4096), (96, 2048, 4097),
    (200, 2100, 7000), (170, 2050, 7003), (4000, 2048, 2051)])
@pytest.mark.parametrize("affine", [False, True], ids=["plain", "affine"])
def test_linear_wgrad_wide(rows, n_in, n_out, dtype, affine):
    """Layers wide enough for the largest tile, with rows that fill none, one
    and several rounds of its steps."""
    test_linear_wgrad(rows, n_in, n_out, dtype, affine)


@TYPES
def test_linear_wgrad_few_outputs_of_many_inputs(dtype):
    for n_out in (1, 7, 9):
        test_linear_wgrad(40, 70001, n_out, dtype, True)


def test_linear_wgrad_bands_share_a_workspace():
    """Bands of falling height, summed with `accumulate`, in the workspace of the
    first one; the choice of splits goes up and down on the way. Nothing is
    written behind it."""
    n_in, n_out, bands = 512, 512, (672, 640, 353, 32, 1)
    tell("wgrad bands", bands)
    rng = np.random.default_rng(5)
    need = L.lrcnn_linear_wgrad_workspace_bytes(bands[0], n_in, n_out, L.BF16)
    assert need > 0
    whole = buf(need + 4096)
    ws = whole[:need]
    dw, db = torch.full((n_out, n_in), 9.0, device="cuda"), torch.full((n_out,), 9.0, device="cuda")
    rw = rb = tw = tb = 0
    for i, rows in enumerate(bands):
        c, q = checkpoint_of(features(rng, rows, n_in))
        dy = matrix(rng.standard_normal((rows, n_out)), BF16)
        L.lrcnn_linear_wgrad(dy, c, dw, ws, db=db, accumulate=i > 0)
        w, b = OB.linear_wgrad(np64(dy), q)
        rw, rb = rw + w, rb + b
        w, b = OB.linear_wgrad(np.abs(np64(dy)), np.abs(q))
        tw, tb = tw + w, tb + b
    close(dw, rw, 1e-5 * tw)
    close(db, rb, 1e-5 * tb)
    assert (whole[need:] == 0xA5).all()


@pytest.mark.parametrize("rows,cols,value", [
    (3, 64, 0.1), (5, 512, 0.1), (70, 96, 0.3), (9, 96, 100.7), (2, 31, -33.3), (4, 1000, 1e-3),
    (3, 2048, 12345.678), (2, 5000, 0.7), (2, 16384, -1e6 / 3)])
def test_layer_norm_of_constant_float32_rows(rows, cols, value):
    """A row of one value has that value as its mean, whatever the rounding of
    its sum, and nothing is left of it but beta: d = v - mean is a few ulps of v,
    a small whole number of them, so its sum and quotient are exact."""
    t = torch.full((rows, cols), value, device="cuda")
    be = torch.randn(cols, device="cuda", generator=torch.Generator("cuda").manual_seed(cols))
    y, c = torch.empty_like(t), ckpt(rows, cols)
    mean, rstd = vec(np.zeros(rows)), vec(np.zeros(rows))
    L.lrcnn_layer_norm_forward(t, None, be, 1e-5, y, mean=mean, rstd=rstd, ckpt=c)
    assert torch.equal(mean, t[:, 0])
    assert torch.equal(y, be.expand(rows, cols))
    # the variance, (d^2) summed less the mean's correction squared: off by 64 u
    # of d^2, d within 64 u of the value
    slack = 64 * 2.0 ** -24 * (64 * 2.0 ** -24 * value) ** 2
    assert np.allclose(np64(rstd), 1e-5 ** -0.5, rtol=1e-6 + slack / 2e-5, atol=0)
    h = torch.empty_like(t)
    L.lrcnn_act8_unpack(c, h)
    assert (h == 0).all()


@pytest.mark.parametrize("cols", [96, 500, 2048, 5000])
def test_layer_norm_far_from_zero(cols):
    """Rows whose mean is 10^4 times their spread: the mean is its float32 value,
    half an ulp off, and the normalised rows carry no more than that plus their
    own 64 u, not the rounding of a sum of large values."""
    rng = np.random.default_rng(cols)
    x = np64(vec(1e4 + rng.standard_normal((40, cols))))
    y, mean, rstd = torch.empty(40, cols, device="cuda"), vec(np.zeros(40)), vec(np.zeros(40))
    L.lrcnn_layer_norm_forward(vec(x), None, None, 1e-5, y, mean=mean, rstd=rstd)
    ry, xh, rm, rr = OB.layer_norm(x, np.ones(cols), 0, 1e-5)
    close(mean, rm, 2.0 ** -24 * np.abs(rm))
    close(rstd, rr, 4e-6 * rr)
    # x - mean0 is exact or off by half its ulp; the correction by 64 u of
    # the mean0's error, itself within 64 u of the mean
    slack = 64 * 2.0 ** -24 * 64 * 2.0 ** -24 * np.abs(rm[:, None])
    close(y, ry, rr[:, None] * slack + 4e-6 * (1 + np.abs(ry)))


@TYPES
@pytest.mark.parametrize("rows,cols", [(4096, 32), (300, 64), (500, 640), (250, 2048), (60, 4096)])
def test_layer_norm_rstd_is_rounded_once(rows, cols, dtype):
    """Rows of a and -a in turn have mean 0 and, for an a of at most 8 bits,
    variance a^2, sums and quotient exact. eps = 0: rstd is the float32 number
    nearest to 1 / a, an error of none in what a whole row is scaled by."""
    a = (128 + np.arange(rows) % 128) * 2.0 ** (np.arange(rows) // 128 % 20 - 15)
    x = a[:, None] * (1 - 2.0 * (np.arange(cols) % 2))
    rstd, y = vec(np.zeros(rows)), torch.empty(rows, cols, device="cuda", dtype=dtype)
    L.lrcnn_layer_norm_forward(matrix(x, dtype), None, None, 0.0, y, rstd=rstd)
    want = (1 / a).astype(np.float32)
    got = rstd.cpu().numpy()
    assert np.array_equal(got, want), f"{(got != want).mean():.2%} of the rows differ"
    # no variance and no eps, a variance past float32, and one that is NaN
    x = np.zeros((3, cols))
    x[1] = 2.0 ** 100 * (1 - 2.0 * (np.arange(cols) % 2))
    x[2, 5] = math.nan
    L.lrcnn_layer_norm_forward(matrix(x, dtype), None, None, 0.0, y[:3], rstd=rstd[:3])
    got = rstd[:3].cpu().numpy()
    assert got[0] == math.inf and got[1] == 0 and np.isnan(got[2])


@TYPES
@pytest.mark.parametrize("e", [-105, -118, -126, -131])
def test_linear_wgrad_of_the_smallest_gradients(e, dtype):
    """Subnormal numbers count. bfloat16 ones exactly; of a float32 dy the three
    pieces keep what 2^-133, the smallest bfloat16 number, can hold, so each value is
    at most 2^-134 off."""
    n = 64
    dy = (1 + np.arange(1, n + 1) * 2.0 ** (-23 if dtype == F32 else -2)) * 2.0 ** e
    t = matrix(np.stack([dy, dy]), dtype)
    d64 = np64(t)
    assert (d64 > 0).all()
    c, q = checkpoint_of(np.full((2, 32), 2.0 ** 40))
    dw, db = torch.empty(n, 32, device="cuda"), torch.empty(n, device="cuda")
    L.lrcnn_linear_wgrad(t, c, dw, db=db)
    off = 2.0 ** -134 if dtype == F32 else 0
    close(dw, d64.T @ q, off * np.abs(q).sum(0) + 2.0 ** -23 * d64.T @ q)
    close(db, d64.sum(0), 2 * off + 2.0 ** -23 * d64.sum(0))
