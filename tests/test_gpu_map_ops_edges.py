"""Calls at the edges of what group norm, dropout and the gated block take: weights and
vectors at an element's alignment, checkpoints of more than 2^32 codes, the widest maps, dropped
shares next to none and all.

Tolerances, u = 2^-24. The gated block: those of its other tests (a sum over a depth D within
D u of its terms' magnitudes, and 8 u for bias and joins; the activation to 4e-6 of its argument,
slopes below 1.2; half an ulp of bfloat16, at most 2^-8 of a value). Rows do not meet, so where a
call's last rows are given to a call of their own that takes the same tile, the bits are the
same. Group norm: y is formed from the returned statistics by (x - mean) rstd, three roundings of
at most |x| + |mean| times rstd, and the checkpoint stands within half a step, step <= 1 / 63.75
of the group's largest; the statistics within 32 u of the largest magnitude and 22 u, and with
long slabs by another u of a running mean and u / 2 for each eight pixels that a thread joins."""
import math

import pytest
import torch

from paper_2401_11471_amd import lrcnn as L
from test_gpu_gated_ffn import BF16, TYPES, U, act, buf, close, product, tile

pytestmark = pytest.mark.gpu


def tell(*a):
    print(*a, flush=True)


def shifted(t, by=1):
    """t, dense, `by` elements behind an aligned address."""
    wide = torch.empty(t.numel() + by, device="cuda", dtype=t.dtype)
    s = wide[by:].view(t.shape)
    s.copy_(t)
    return s


@TYPES
@pytest.mark.parametrize("variant", [-1, 0, 2, 3, 4, 5, 6])
@pytest.mark.parametrize("rows,n,hidden", [(7, 72, 40), (290, 72, 264), (270, 33, 65)])
def test_gated_weights_at_an_elements_alignment(rows, n, hidden, variant, dtype, tile):
    tell("weights", rows, n, hidden, variant, dtype)
    tile(variant)
    g = torch.Generator(device="cuda").manual_seed(rows)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x, dz = r(rows, n).to(dtype), r(rows, n).to(dtype)
    w1 = shifted((r(2 * hidden, n) / math.sqrt(n)).to(dtype))
    w2 = shifted((r(n, hidden) / math.sqrt(hidden)).to(dtype))
    b1, b2 = shifted(r(2 * hidden)), shifted(r(n))
    e = lambda w: torch.empty(rows, w, device="cuda", dtype=dtype)
    a, z, uv, duv, dx = e(hidden), e(n), e(2 * hidden), e(2 * hidden), e(n)
    L.lrcnn_gated_ffn_forward(L.ACT_SILU, x, w1, a, b1, w2, b2, z, uv)
    ruv, err = product(x, w1, b1)
    (u, v), (eu, ev) = ruv.chunk(2, 1), err.chunk(2, 1)
    f = act(u, "silu")[0]
    close(uv, ruv, err, dtype)
    close(a, f * v, (1.2 * eu + 4e-6 * u.abs()) * (v.abs() + ev) + f.abs() * ev
          + 2 * U * (f * v).abs(), dtype)
    close(z, *product(a, w2, b2), dtype)
    w2t, w1t = shifted(w2.t().contiguous()), shifted(w1.t().contiguous())
    L.lrcnn_gated_ffn_backward(L.ACT_SILU, dz, w2t, duv, uv, w1t=w1t, dx=dx)
    u, v = uv.double().chunk(2, 1)
    da, err = product(dz, w2t)
    f, df = act(u, "silu")
    ef = 4e-6 * (1 + u.abs()) + 2 * U
    close(duv[:, :hidden], da * df * v, v.abs() * (err * 1.2 + da.abs() * (ef + 4 * U)), dtype)
    close(duv[:, hidden:], da * f, err * f.abs() + (da.abs() + err) * (4e-6 * u.abs()
                                                                       + 2 * U * f.abs()), dtype)
    close(dx, *product(duv, w1t), dtype)


@pytest.mark.parametrize("variant", [0, 2, 4])
def test_gated_checkpoints_past_32_bits(variant, tile):
    """More than 2^32 codes in each checkpoint, by tiles that copy codes, and that read them."""
    rows, n, hidden, last = (1 << 19) + 8500, 64, 8192, 768
    tell("gated checkpoints past 32 bits", variant)
    assert rows * hidden > 1 << 32 and rows % 256 != 0
    tile(variant)
    g = torch.Generator(device="cuda").manual_seed(variant)
    r = lambda *s: (torch.randn(*s, generator=g, device="cuda") / 8).bfloat16()
    x, w1, w2t = r(rows, n), r(2 * hidden, n), r(hidden, n)
    b1 = torch.randn(2 * hidden, generator=g, device="cuda")
    # (the last rows begin where a tile does)
    first = (rows - last) // 256 * 256
    ku, kv, ka = (buf(rows, hidden) for _ in range(3))
    a = torch.empty(rows, hidden, device="cuda", dtype=BF16)
    L.lrcnn_gated_ffn_forward(L.ACT_SILU, x, w1, a, b1, ckpt_u=ku, ckpt_v=kv)
    some = rows - first
    k = [buf(some, hidden) for _ in range(3)]
    a2 = torch.empty(some, hidden, device="cuda", dtype=BF16)
    L.lrcnn_gated_ffn_forward(L.ACT_SILU, x[first:], w1, a2, b1, ckpt_u=k[0], ckpt_v=k[1])
    assert torch.equal(a[first:], a2)
    del a, a2
    duv = torch.empty(rows, 2 * hidden, device="cuda", dtype=BF16)
    L.lrcnn_gated_ffn_backward(L.ACT_SILU, x, w2t, duv, ckpt_u=ku, ckpt_v=kv, ckpt_a=ka)
    duv2 = torch.empty(some, 2 * hidden, device="cuda", dtype=BF16)
    L.lrcnn_gated_ffn_backward(L.ACT_SILU, x[first:], w2t, duv2, ckpt_u=k[0], ckpt_v=k[1],
                               ckpt_a=k[2])
    assert torch.isfinite(duv2).all() and torch.equal(duv[first:], duv2)
    codes, groups = some * hidden, some * (hidden // 32)
    for big, small in zip((ku, kv, ka), k):
        assert torch.equal(big[first * hidden:rows * hidden], small[:codes])
        assert torch.equal(big[rows * hidden:][first * (hidden // 32):rows * (hidden // 32)],
                           small[codes:][:groups])


@pytest.mark.parametrize("batch,pixels,groups", [(233100, 9, 8), (2, 1050000, 32)])
def test_group_norm_checkpoints_past_32_bits(batch, pixels, groups):
    """Maps in one block, and in slabs, whose checkpoint has more than 2^32 codes: the last rows
    of y and of the checkpoint, then dx from that checkpoint."""
    cols, last = 2048, 9
    tell("group norm checkpoints past 32 bits", batch, pixels)
    rows = batch * pixels
    assert rows * cols > 1 << 32
    g = torch.Generator(device="cuda").manual_seed(pixels)
    x = torch.empty(rows, cols, device="cuda", dtype=BF16).normal_(generator=g)
    y, ck = torch.empty_like(x), buf(rows, cols)
    ws = torch.empty(L.lrcnn_group_norm_workspace_bytes(batch, pixels, cols, groups), device="cuda",
                     dtype=torch.uint8)
    mean, rstd = (torch.empty(batch, groups, device="cuda") for _ in range(2))
    L.lrcnn_group_norm_forward(L.ACT_NONE, x, None, None, 1e-5, y, batch, groups, ws, mean, rstd, ck)

    def image(t, f):
        """Sums over the last image's groups of f(rows of t), in float64."""
        s = 0
        for part in t[rows - pixels:].split(1 << 17):
            s = s + f(part.double()).view(-1, groups, cols // groups).sum((0, 2))
        return s / (pixels * (cols // groups))
    wide = lambda s: s.double().repeat_interleave(cols // groups)
    m = image(x, lambda p: p)
    var = image(x, lambda p: (p - wide(m)) ** 2)
    # (a slab of two images: 1 / 256 of the pixels, a quarter of them a thread's; no value of the
    # normal reaches 8, no mean of eight 4)
    joins = pixels / 256 / 4 / 8
    assert ((mean[-1] - m).abs() <= (32 * 8 + joins * 4) * U).all()
    assert ((rstd[-1] * (var + 1e-5).sqrt() - 1).abs() <= (22 + joins / 2) * U).all()
    X, M, R = x[-last:].double(), wide(mean[-1]), wide(rstd[-1])
    xh = (X - M) * R
    err = 3 * U * (X.abs() + M.abs()) * R
    close(y[-last:], xh, err, BF16)
    # the checkpoint's last rows, as a checkpoint of their own
    codes = ck[(rows - last) * cols:rows * cols].view(torch.int8).view(last, cols).double()
    e = ck[rows * cols:][(rows - last) * (cols // 32):rows * (cols // 32)].view(last, -1).double()
    k = codes * torch.exp2(e - 133).repeat_interleave(32, 1)
    top = (xh.abs() + err).view(last, -1, 32).amax(2).repeat_interleave(32, 1)
    assert ((k - xh).abs() <= 0.5 * top / 63.75 + err).all()
    # backward, dy in y's place: dx = rstd (dy - mean(dy) - xh mean(dy xh)), xh as held
    held_rows = ck[:rows * cols].view(torch.int8).view(rows, cols)
    exps = ck[rows * cols:rows * cols + rows * (cols // 32)].view(rows, cols // 32)
    s1 = s2 = a1 = a2 = 0
    for i in range(rows - pixels, rows, 1 << 17):
        j = min(i + (1 << 17), rows)
        d = y[i:j].double()
        h = held_rows[i:j].double() * torch.exp2(exps[i:j].double() - 133).repeat_interleave(32, 1)
        add = lambda t: t.view(-1, groups, cols // groups).sum((0, 2)) / (pixels * (cols // groups))
        s1, s2 = s1 + add(d), s2 + add(d * h)
        a1, a2 = a1 + add(d.abs()), a2 + add((d * h).abs())
    dy = y[-last:].double()
    L.lrcnn_group_norm_backward(L.ACT_NONE, y, rstd, None, None, y, batch, groups, ws, ckpt=ck)
    dx = R * (dy - wide(s1) - k * wide(s2))
    # a thread adds a slab's rows one after the other: at most (slab / 4 + 16) u of the terms,
    # a slab being at most 4 times the image over 2048, or a thread's 8 pixels
    adds = (max(4 * pixels / 2048, 8) / 4 + 16) * U
    tol = R * (wide(a1) * adds + k.abs() * wide(a2) * adds
               + 4 * U * (dy.abs() + wide(s1).abs() + 2 * (k * wide(s2)).abs()))
    close(y[-last:], dx, tol, BF16)


@TYPES
@pytest.mark.parametrize("batch,pixels,groups", [(3, 5, 1), (2, 3, 1 << 19), (1, 40, 1 << 10)])
def test_group_norm_of_the_widest_maps(batch, pixels, groups, dtype):
    cols = 1 << 20
    tell("widest", batch, pixels, groups, dtype)
    rows = batch * pixels
    g = torch.Generator(device="cuda").manual_seed(groups)
    x, dy = (torch.randn(rows, cols, generator=g, device="cuda").to(dtype) for _ in range(2))
    y, dx = torch.empty_like(x), torch.empty_like(x)
    ws = torch.empty(L.lrcnn_group_norm_workspace_bytes(batch, pixels, cols, groups), device="cuda",
                     dtype=torch.uint8)
    mean, rstd = (torch.empty(batch, groups, device="cuda") for _ in range(2))
    dg, db = torch.empty(2, cols, device="cuda").unbind(0)
    L.lrcnn_group_norm_forward(L.ACT_NONE, x, None, None, 1e-3, y, batch, groups, ws, mean, rstd)
    L.lrcnn_group_norm_backward(L.ACT_NONE, dy, rstd, None, None, dx, batch, groups, ws, dgamma=dg,
                                dbeta=db, x=x, mean=mean)
    by = lambda t: t.double().view(batch, pixels, groups, -1)
    at = lambda s: s.double()[:, None, :, None]
    X = by(x)
    m = X.mean((1, 3))
    r = 1 / ((X - at(m)).square().mean((1, 3)) + float(torch.tensor(1e-3))).sqrt()
    top = X.abs().amax((1, 3))
    assert ((mean - m).abs() <= 32 * U * top).all() and ((rstd / r - 1).abs() <= 22 * U).all()
    xh = (X - at(mean)) * at(rstd)
    err = 3 * U * (X.abs() + at(mean).abs()) * at(rstd)
    flat = lambda t: t.reshape(rows, cols)
    close(y, flat(xh), flat(err), dtype)
    # sums of at most 40 pixels in float32, channels in 64 bits: 40 u, xh itself within err
    d = by(dy)
    close(db, flat(d).sum(0), 42 * U * flat(d).abs().sum(0))
    close(dg, flat(d * xh).sum(0), flat(d.abs() * (err + 42 * U * xh.abs())).sum(0))
    m1, m2 = d.mean((1, 3), True), (d * xh).mean((1, 3), True)
    a1 = d.abs().mean((1, 3), True)
    a2 = (d.abs() * (err + 42 * U * xh.abs())).mean((1, 3), True)
    tol = at(rstd) * (42 * U * a1 + xh.abs() * a2 + err * m2.abs()
                      + 4 * U * (d.abs() + m1.abs() + 2 * (xh * m2).abs()))
    close(dx, flat(at(rstd) * (d - m1 - xh * m2)), flat(tol), dtype)


@TYPES
def test_dropout_next_to_none_and_all(dtype):
    """rint(65536 p) is what counts: 0 below 2^-17, all from 1 - 2^-17 on, ties to even."""
    g = torch.Generator(device="cuda").manual_seed(4)
    x, res = (torch.randn(50, 333, generator=g, device="cuda").to(dtype) for _ in range(2))
    y, state = torch.empty_like(x), torch.tensor([-1, -2], device="cuda")
    for p in (0.0, 2.0 ** -18, 2.0 ** -17):
        L.lrcnn_dropout(x, y, p, state)
        assert torch.equal(y, x), p
    for p in (1.0, 1 - 2.0 ** -18, 1 - 2.0 ** -17):
        L.lrcnn_dropout(x, y, p, state, residual=res)
        assert torch.equal(y, res), p
        L.lrcnn_dropout(torch.full_like(x, math.nan), y, p, state)
        assert (y == 0).all(), p


def test_dropout_of_the_widest_rows():
    """A row of 2^30 - 5 columns (its last vector cut): counters past 2^27."""
    cols = (1 << 30) - 5
    tell("dropout of the widest rows")
    from oracle import map_ops as OM
    x = torch.ones(1, cols, device="cuda", dtype=BF16)
    y, state = torch.empty_like(x), torch.tensor([6, 7], device="cuda")
    L.lrcnn_dropout(x, y, 0.5, state)
    # a row's last columns draw what the first of a matrix of one vector a row draw there
    at = cols // 8 - 100
    bits = OM.dropout_bits(6, 7, 101, 8, first_row=at).reshape(-1)[:cols - 8 * at]
    want = torch.from_numpy((bits >= 32768) * 2.0).cuda()
    assert torch.equal(y[0, 8 * at:].double(), want)
