"""The gated feed-forward block on the GPU against its formulas in float64: from one
row and one feature on, every kernel variant (few rows, small, middle and large tiles,
operands that are not aligned), slices with odd strides, checkpoints, values that
are not finite, graphs.

Tolerances, with u = 2^-24 (float32 rounding). A sum over a depth of D is off by at most
D u times the sum S of the magnitudes (products of bfloat16 are exact, float32's fused);
bias and the splits' joins add 8 roundings. f(u) is evaluated to 4e-6 of u, slopes below
1.2. Products with stored results (a, du and dv) are checked on what was stored. A
bfloat16 result adds half an ulp, 2^-9 of the value, taken as 2^-8 where the value
itself is uncertain by the float32 error. A checkpoint stands within half its step."""
import math

import pytest
import torch

from paper_2401_11471_amd import lrcnn as L

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
TYPES = pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
KINDS = {"relu": L.ACT_RELU, "gelu": L.ACT_GELU, "gelu_tanh": L.ACT_GELU_TANH, "silu": L.ACT_SILU}
# rows, n_in, hidden, n_out
SHAPES = [(1, 1, 1, 1), (1, 8, 7, 5), (2, 64, 32, 64), (1, 1000, 130, 40), (16, 72, 64, 72),
          (17, 128, 100, 33), (32, 520, 40, 264), (33, 64, 64, 64), (5, 33, 31, 30), (65, 40, 33, 16),
          (130, 136, 96, 200), (300, 37, 77, 51), (64, 1032, 65, 8), (257, 16, 300, 24)]
# (as many tiles as make the middle and the large one)
WIDE = [(2100, 72, 1000, 1040), (2100, 70, 1001, 1030), (4200, 72, 2080, 1100)]


def tell(*a):
    print(*a, flush=True)


def matrix(t, dtype, pad=0, at=0):
    """t in `dtype`; pad > 0: a slice of a wider matrix from column `at`, NaN around it."""
    if not pad:
        return t.to(dtype).contiguous()
    rows, cols = t.shape
    wide = torch.full((rows, cols + pad), math.nan, device="cuda", dtype=dtype)
    s = wide[:, at:at + cols]
    s.copy_(t)
    return s


def untouched(s, at):
    cols = s.shape[1]
    assert torch.isnan(s._base[:, :at]).all() and torch.isnan(s._base[:, at + cols:]).all()


def buf(rows, cols):
    return torch.full((L.lrcnn_act8_bytes(rows, cols),), 0xA5, device="cuda", dtype=torch.uint8)


def act(u, kind):
    """f and f' in float64."""
    if kind == "relu":
        return u.clamp_min(0), (u > 0).double()
    if kind == "silu":
        s = torch.sigmoid(u)
        return u * s, s + u * s * (1 - s)
    if kind == "gelu":
        phi = torch.special.ndtr(u)
        return u * phi, phi + u * torch.exp(-u * u / 2) / math.sqrt(2 * math.pi)
    k = math.sqrt(2 / math.pi)
    s = torch.sigmoid(2 * k * (u + 0.044715 * u ** 3))
    return u * s, s + u * s * (1 - s) * 2 * k * (1 + 3 * 0.044715 * u * u)


def close(got, ref, tol, dtype=F32):
    got = got.double()
    assert got.shape == ref.shape and torch.isfinite(got).all()
    over = (got - ref).abs() - (tol + ref.abs() * (2.0 ** -8 if dtype == BF16 else 0) + 1e-37)
    assert (over <= 0).all(), f"off by {(got - ref).abs().max():.3g}, {over.max():.3g} over"


def held(ckpt, rows, cols):
    y = torch.empty(rows, cols, device="cuda")
    L.lrcnn_act8_unpack(ckpt, y)
    return y.double()


def held_close(ckpt, ref, err):
    """A checkpoint's values against the full ones, known to err: half a step. For a
    largest magnitude m in [2^p, 2^(p+1)) the step is 2^(p-6) <= m / 64 or, from
    m = 127.5 2^(p-6) on, 2^(p-5) <= m / 63.75. (The codes of the columns behind the
    last are zero.)"""
    rows, cols = ref.shape
    pitch = -(-cols // 32) * 32
    wide = torch.nn.functional.pad(ref.abs() + err, (0, pitch - cols)).view(rows, -1, 32)
    step = (wide.amax(2, True) / 63.75).expand(wide.shape).reshape(rows, pitch)[:, :cols]
    assert ((held(ckpt, rows, cols) - ref).abs() <= 0.5 * step + err + 2.0 ** -127).all()
    codes = ckpt[:rows * pitch].view(rows, pitch)
    assert (codes[:, cols:] == 0).all()


def product(x, w, bias=None):
    """x w^T + bias in float64 and its error's bound."""
    x, w = x.double(), w.double()
    y, s = x @ w.t(), x.abs() @ w.abs().t()
    if bias is not None:
        y, s = y + bias.double(), s + bias.double().abs()
    return y, (x.shape[1] + 8) * U * s


def case(rows, n_in, hidden, n_out, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")
    return n, dict(x=n(rows, n_in), w1=(n(2 * hidden, n_in) / math.sqrt(n_in)).to(dtype),
                   b1=0.2 * n(2 * hidden), w2=(n(n_out, hidden) / math.sqrt(hidden)).to(dtype),
                   b2=0.2 * n(n_out))


def check_forward(rows, n_in, hidden, n_out, dtype, kind, pad, at, ckpts, full, bias=True):
    tell("gated forward", rows, n_in, hidden, n_out, dtype, kind, pad, ckpts, full)
    _, s = case(rows, n_in, hidden, n_out, dtype, rows + hidden)
    x, w1, w2 = matrix(s["x"], dtype, pad, at), s["w1"], s["w2"]
    b1, b2 = (s["b1"], s["b2"]) if bias else (None, None)
    out = lambda w: matrix(torch.zeros(rows, w, device="cuda"), dtype, pad, at)
    a, z = out(hidden), out(n_out)
    uv = out(2 * hidden) if full else None
    ku, kv = (buf(rows, hidden), buf(rows, hidden)) if ckpts else (None, None)
    L.lrcnn_gated_ffn_forward(KINDS[kind], x, w1, a, b1=b1, w2=w2, b2=b2, z=z, uv=uv, ckpt_u=ku,
                              ckpt_v=kv)
    ruv, err = product(x, w1, b1)
    u, v, eu, ev = ruv[:, :hidden], ruv[:, hidden:], err[:, :hidden], err[:, hidden:]
    f = act(u, kind)[0]
    ea = (1.2 * eu + 4e-6 * u.abs()) * (v.abs() + ev) + f.abs() * ev + 2 * U * (f * v).abs()
    close(a, f * v, ea, dtype)
    close(z, *product(a, w2, b2), dtype)
    if full:
        close(uv, ruv, err, dtype)
    if ckpts:
        held_close(ku, u, eu)
        held_close(kv, v, ev)
    if pad:
        for t in (a, z) + ((uv,) if full else ()):
            untouched(t, at)
    # without z: the same a
    a2 = torch.empty(rows, hidden, device="cuda", dtype=dtype)
    L.lrcnn_gated_ffn_forward(KINDS[kind], x, w1, a2, b1=b1, ckpt_u=ku, ckpt_v=kv)
    assert torch.equal(a, a2)


def check_backward(rows, n_in, hidden, n_out, dtype, kind, pad, at, saved):
    tell("gated backward", rows, n_in, hidden, n_out, dtype, kind, pad, saved)
    n, s = case(rows, n_in, hidden, n_out, dtype, rows * 3 + hidden)
    dz = matrix(n(rows, n_out), dtype, pad, at)
    uv = n(rows, 2 * hidden)
    w2t, w1t = s["w2"].t().contiguous(), s["w1"].t().contiguous()
    duv = matrix(torch.zeros(rows, 2 * hidden, device="cuda"), dtype, pad, at)
    dx = matrix(torch.zeros(rows, n_in, device="cuda"), dtype, pad, at)
    if saved:
        ku, kv, ka = (buf(rows, hidden) for _ in range(3))
        L.lrcnn_act8_pack(uv[:, :hidden], ku)
        L.lrcnn_act8_pack(uv[:, hidden:], kv)
        kw = dict(ckpt_u=ku, ckpt_v=kv, ckpt_a=ka)
        u, v = held(ku, rows, hidden), held(kv, rows, hidden)
    else:
        uv = matrix(uv, dtype, pad, at)
        kw, ka = dict(uv=uv), None
        u, v = uv[:, :hidden].double(), uv[:, hidden:].double()
    L.lrcnn_gated_ffn_backward(KINDS[kind], dz, w2t, duv, w1t=w1t, dx=dx, **kw)
    da, err = product(dz, w2t)
    f, df = act(u, kind)
    ef = 4e-6 * (1 + u.abs()) + 2 * U
    close(duv[:, :hidden], da * df * v, v.abs() * (err * 1.2 + da.abs() * (ef + 4 * U)), dtype)
    close(duv[:, hidden:], da * f, err * f.abs() + (da.abs() + err) * (4e-6 * u.abs() + 2 * U * f.abs()),
          dtype)
    close(dx, *product(duv, w1t), dtype)
    if saved:
        held_close(ka, f * v, (4e-6 * u.abs() + 2 * U * f.abs()) * v.abs())
    if pad:
        untouched(duv, at)
        untouched(dx, at)
    # without dx, and in place of uv: the same
    again = torch.empty(rows, 2 * hidden, device="cuda", dtype=dtype) if saved else uv
    L.lrcnn_gated_ffn_backward(KINDS[kind], dz, w2t, again, **kw)
    assert torch.equal(again, duv)


@TYPES
@pytest.mark.parametrize("rows,n_in,hidden,n_out", SHAPES)
def test_forward(rows, n_in, hidden, n_out, dtype):
    for i, kind in enumerate(KINDS):
        pad, at = [(0, 0), (3, 1), (8, 8), (16, 0)][i]
        check_forward(rows, n_in, hidden, n_out, dtype, kind, pad, at, ckpts=i in (0, 3),
                      full=i in (1, 3), bias=i != 2)
    check_forward(rows, n_in, hidden, n_out, dtype, "silu", 0, 0, False, True)


@TYPES
@pytest.mark.parametrize("rows,n_in,hidden,n_out", SHAPES)
def test_backward(rows, n_in, hidden, n_out, dtype):
    for i, kind in enumerate(KINDS):
        pad, at = [(0, 0), (3, 1), (8, 8), (16, 0)][i]
        for saved in (False, True):
            check_backward(rows, n_in, hidden, n_out, dtype, kind, pad, at, saved)


@TYPES
@pytest.mark.parametrize("rows,n_in,hidden,n_out", WIDE)
def test_wide(rows, n_in, hidden, n_out, dtype):
    check_forward(rows, n_in, hidden, n_out, dtype, "silu", 0, 0, True, True)
    check_forward(rows, n_in, hidden, n_out, dtype, "gelu", 8, 8, True, False)
    check_backward(rows, n_in, hidden, n_out, dtype, "silu", 0, 0, True)
    check_backward(rows, n_in, hidden, n_out, dtype, "relu", 8, 8, False)


@pytest.fixture
def tile():
    """Takes a variant of the products, and leaves the choice to the library after."""
    yield L.lrcnn_debug_ffn_tile
    L.lrcnn_debug_ffn_tile(-1)


@TYPES
@pytest.mark.parametrize("variant", range(8))
def test_every_tile(variant, dtype, tile):
    """Each variant at sizes that end inside its tiles, in one step and in many, aligned
    and not, from checkpoints and full-width values."""
    tile(variant)
    tell("tile", variant)
    for rows, n_in, hidden, n_out in [(300, 200, 152, 136), (130, 64, 288, 264), (33, 328, 40, 72)]:
        if variant == 7:
            rows = 29 if rows > 100 else 11
        check_forward(rows, n_in, hidden, n_out, dtype, "silu", 0, 0, True, True)
        check_forward(rows, n_in, hidden, n_out, dtype, "gelu_tanh", 8, 8, variant != 7, False)
        check_backward(rows, n_in, hidden, n_out, dtype, "silu", 0, 0, True)
        check_backward(rows, n_in, hidden, n_out, dtype, "gelu", 8, 8, False)
    rows = 21 if variant == 7 else 270
    check_forward(rows, 77, 129, 65, dtype, "relu", 3, 1, True, True)
    check_backward(rows, 77, 129, 65, dtype, "silu", 3, 1, True)


@TYPES
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("variant", [0, 1])
def test_whole_and_cut_strips(variant, kind, dtype, tile):
    """Wide tiles with strips that are whole and that end early, rows and features, by kind."""
    tile(variant)
    for rows, n_in, hidden, n_out in [(300, 72, 200, 136), (260, 64, 256, 64)]:
        check_forward(rows, n_in, hidden, n_out, dtype, kind, 8, 8, True, True)
        check_backward(rows, n_in, hidden, n_out, dtype, kind, 8, 8, True)
        check_backward(rows, n_in, hidden, n_out, dtype, kind, 8, 8, False)


@pytest.mark.parametrize("variant", range(8))
def test_groups_that_are_not_finite(variant, tile):
    """A checkpoint's group that stands for NaN: its columns alone are spoiled, and the
    checkpoint of a has NaN for the group; the type's largest values are held."""
    tile(variant)
    rows, n_in, hidden, n_out = (20 if variant == 7 else 300), 40, 200, 72
    tell("groups", variant)
    n, s = case(rows, n_in, hidden, n_out, F32, 6)
    u, v, dz = n(rows, hidden), n(rows, hidden), n(rows, n_out)
    w2t = s["w2"].t().contiguous()
    results = []
    for bad in (False, True):
        if bad:
            u[3, 70], v[5, 10] = math.nan, -math.inf
            v[7, 130] = torch.finfo(F32).max
        ku, kv, ka = (buf(rows, hidden) for _ in range(3))
        L.lrcnn_act8_pack(u, ku)
        L.lrcnn_act8_pack(v, kv)
        duv = torch.empty(rows, 2 * hidden, device="cuda")
        L.lrcnn_gated_ffn_backward(L.ACT_GELU, dz, w2t, duv, ckpt_u=ku, ckpt_v=kv, ckpt_a=ka)
        results.append((duv, held(ka, rows, hidden), held(kv, rows, hidden)))
    (good, ga, _), (got, a, hv) = results
    spoiled = torch.zeros(rows, hidden, dtype=torch.bool, device="cuda")
    spoiled[3, 64:96] = spoiled[5, :32] = spoiled[7, 128:160] = True
    du, dv = got.chunk(2, 1)
    assert torch.isnan(du[3, 64:96]).all() and torch.isnan(dv[3, 64:96]).all()
    assert torch.isnan(du[5, :32]).all() and torch.isnan(a[5, :32]).all()
    assert torch.equal(dv[5], good.chunk(2, 1)[1][5])      # dv has no v
    assert torch.isnan(a[3, 64:96]).all()
    assert hv[7, 130] == 127 * 2.0 ** 121                  # the top binade's last step
    assert not torch.isnan(du[7]).any() and not torch.isnan(a[7]).any()
    keep = ~spoiled
    for p, q in zip((du, dv), good.chunk(2, 1)):
        assert torch.equal(p[keep], q[keep])
    assert torch.equal(a[keep], ga[keep])


@pytest.mark.parametrize("variant", range(8))
def test_rows_do_not_meet(variant, tile):
    """A row that is not finite spoils its own results alone, in every variant."""
    tile(variant)
    for rows, n_in, hidden, n_out in [(20, 64, 48, 40), (300, 72, 200, 264)]:
        tell("rows", variant, rows, n_in, hidden, n_out)
        _, s = case(rows, n_in, hidden, n_out, BF16, 5)
        x = s["x"].bfloat16()
        run = lambda: (torch.empty(rows, hidden, device="cuda", dtype=BF16),
                       torch.empty(rows, n_out, device="cuda", dtype=BF16), buf(rows, hidden))
        good, bad = run(), run()
        bads = [3, rows - 1]
        for i, (a, z, k) in enumerate((good, bad)):
            if i:
                x[bads[0], 5], x[bads[1], 1] = math.nan, math.inf
            L.lrcnn_gated_ffn_forward(L.ACT_SILU, x, s["w1"], a, s["b1"], w2=s["w2"], b2=s["b2"], z=z,
                                      ckpt_u=k)
        keep = torch.ones(rows, dtype=torch.bool, device="cuda")
        keep[bads] = False
        for p, q in zip(good[:2], bad[:2]):
            assert torch.equal(p[keep], q[keep]) and torch.isfinite(p).all()
            assert not torch.isfinite(q[bads]).any()
        assert torch.equal(held(good[2], rows, hidden)[keep], held(bad[2], rows, hidden)[keep])
        assert torch.isnan(held(bad[2], rows, hidden)[bads[0]]).all()


@TYPES
def test_by_differences(dtype):
    """dx against differences of the forward kernels in float32, 2 eps = 2^-5 apart
    (their own error some 1e-3 of the terms); bfloat16: the same weights' dx from the
    float32 chain within four roundings of 2^-9 on the way."""
    rows, n_in, hidden, n_out = 6, 10, 12, 9
    n, s = case(rows, n_in, hidden, n_out, F32, 3)
    if dtype == BF16:
        s = {k: v.bfloat16().float() if k != "b1" and k != "b2" else v for k, v in s.items()}
    dz = n(rows, n_out).to(dtype).float()

    def forward(x):
        a, z = torch.empty(rows, hidden, device="cuda"), torch.empty(rows, n_out, device="cuda")
        uv = torch.empty(rows, 2 * hidden, device="cuda")
        L.lrcnn_gated_ffn_forward(L.ACT_GELU_TANH, x, s["w1"], a, s["b1"], s["w2"], s["b2"], z, uv)
        return float((z.double() * dz.double()).sum()), uv
    _, uv = forward(s["x"])
    dx = torch.empty(rows, n_in, device="cuda", dtype=dtype)
    duv = torch.empty(rows, 2 * hidden, device="cuda", dtype=dtype)
    t = lambda w: w.t().contiguous().to(dtype)
    L.lrcnn_gated_ffn_backward(L.ACT_GELU_TANH, dz.to(dtype), t(s["w2"]), duv, uv.to(dtype),
                               w1t=t(s["w1"]), dx=dx)
    eps, worst, top = 2.0 ** -6, 0.0, float(dx.abs().max())
    for i in range(0, rows * n_in, 3):
        x = s["x"].clone()
        x.view(-1)[i] += eps
        hi = forward(x)[0]
        x.view(-1)[i] -= 2 * eps
        lo = forward(x)[0]
        worst = max(worst, abs((hi - lo) / (2 * eps) - float(dx.view(-1)[i])))
    assert worst < top * (5e-3 if dtype == F32 else 3e-2)


@TYPES
@pytest.mark.parametrize("rows", [5, 33, 300, 2100])
def test_in_place(rows, dtype):
    """z over x, duv over uv, dx over dz, or over uv where duv is elsewhere; the
    checkpoint of a over u's: the same as apart."""
    tell("gated in place", rows, dtype)
    n = 264
    _, s = case(rows, n, n // 2, n, dtype, 12)
    x, w2t, w1t = s["x"].to(dtype), s["w2"].t().contiguous(), s["w1"].t().contiguous()
    a, uv = (torch.empty(rows, w, device="cuda", dtype=dtype) for w in (n // 2, n))
    ku, kv, ka = (buf(rows, n // 2) for _ in range(3))
    z, duv, dx = torch.empty_like(x), torch.empty_like(uv), torch.empty_like(x)
    weights = s["w1"], a, s["b1"], s["w2"], s["b2"]
    L.lrcnn_gated_ffn_forward(L.ACT_SILU, x, *weights, z, uv, ku, kv)
    t = x.clone()
    L.lrcnn_gated_ffn_forward(L.ACT_SILU, t, *weights, t)
    assert torch.equal(t, z)
    for held in (dict(ckpt_u=ku, ckpt_v=kv), dict(uv=uv)):
        L.lrcnn_gated_ffn_backward(L.ACT_SILU, x, w2t, duv, ckpt_a=ka, w1t=w1t, dx=dx, **held)
        t, o = x.clone(), torch.empty_like(duv)
        mine = {k: v.clone() for k, v in held.items()}
        if "uv" in held:
            o = mine["uv"]
            k = torch.empty_like(ka)
        else:
            k = mine["ckpt_u"]
        L.lrcnn_gated_ffn_backward(L.ACT_SILU, t, w2t, o, ckpt_a=k, w1t=w1t, dx=t, **mine)
        assert torch.equal(t, dx) and torch.equal(o, duv)
        g = (n // 2 + 31) // 32 * 32 * rows
        assert torch.equal(k[:g], ka[:g])
    mine = uv.clone()
    L.lrcnn_gated_ffn_backward(L.ACT_SILU, x, w2t, duv, mine, w1t=w1t, dx=mine)
    assert torch.equal(mine, dx)


def test_no_rows():
    x, w = torch.empty(0, 16, device="cuda"), torch.zeros(32, 16, device="cuda")
    k = torch.empty(0, device="cuda", dtype=torch.uint8)
    L.lrcnn_gated_ffn_forward(L.ACT_SILU, x, w, x, ckpt_u=k, ckpt_v=k)
    d = torch.empty(0, 32, device="cuda")
    L.lrcnn_gated_ffn_backward(L.ACT_SILU, x, w[:16], d, uv=d)


def test_past_32_bits():
    """Rows of every operand more than 2^32 bytes from the first."""
    rows, n_in, hidden, n_out, ld = 4400, 64, 96, 64, 1 << 20
    tell("gated past 32 bits")
    _, s = case(rows, n_in, hidden, n_out, BF16, 9)
    wide = torch.empty(rows, ld, device="cuda", dtype=BF16)
    at = lambda c, w: wide[:, c:c + w]
    x, a, z, uv, dz, dx = (at(1024 * i, w) for i, w in enumerate(
        (n_in, hidden, n_out, 2 * hidden, n_out, n_in)))
    x.copy_(s["x"])
    dz.copy_(s["x"] * 0.5)
    w2t, w1t = s["w2"].t().contiguous(), s["w1"].t().contiguous()

    def run(x, a, z, uv, dz, dx):
        L.lrcnn_gated_ffn_forward(L.ACT_SILU, x, s["w1"], a, s["b1"], s["w2"], s["b2"], z, uv)
        L.lrcnn_gated_ffn_backward(L.ACT_SILU, dz, w2t, uv, uv, w1t=w1t, dx=dx)
    run(x, a, z, uv, dz, dx)
    d = [torch.empty_like(t, memory_format=torch.contiguous_format) for t in (a, z, uv)]
    dxd = torch.empty(rows, n_in, device="cuda", dtype=BF16)
    run(x.contiguous(), *d, dz.contiguous(), dxd)
    for p, q in zip((a, z, uv, dx), (*d, dxd)):
        assert torch.equal(p, q)


def test_far_weights_in_many_tiles():
    """Weights of 4 GiB, past the wide tiles' offsets, and more than 2^22 tiles of 64 x 64."""
    rows, n_in, hidden = 1030, 128, 1 << 23
    tell("gated far weights")
    g = torch.Generator("cuda").manual_seed(11)
    x = torch.randn(rows, n_in, device="cuda", generator=g).bfloat16()
    w = torch.empty(2 * hidden, n_in, device="cuda", dtype=BF16).normal_(0, 0.3, generator=g)
    a = torch.full((rows, hidden), math.nan, device="cuda", dtype=BF16)
    L.lrcnn_gated_ffn_forward(L.ACT_SILU, x, w, a)
    r = torch.cat([torch.randint(rows, (4000,), generator=g, device="cuda"),
                   torch.tensor([0, rows - 1], device="cuda").repeat(2)])
    f = torch.cat([torch.randint(hidden, (4000,), generator=g, device="cuda"),
                   torch.tensor([0, 0, hidden - 1, hidden - 1], device="cuda")])
    X, wu, wv = x[r].double(), w[f].double(), w[f + hidden].double()
    u, v = (X * wu).sum(1), (X * wv).sum(1)
    eu, ev = ((n_in + 8) * U * (X * t).abs().sum(1) for t in (wu, wv))
    fu, _ = act(u, "silu")
    error = (1.2 * eu + 4e-6 * u.abs()) * (v.abs() + ev) + fu.abs() * ev
    assert ((a[r, f].double() - fu * v).abs() <= 2.0 ** -8 * (fu * v).abs() + 1.01 * error).all()


@TYPES
def test_in_a_graph_and_on_a_stream(dtype):
    """A captured forward and backward pass, on another stream than the tensors' own;
    every replay, with eager work between, equals the eager result."""
    for rows in (3, 200):
        n_in, hidden, n_out = 64, 96, 64
        n, s = case(rows, n_in, hidden, n_out, dtype, 7)
        x, dz = s["x"].to(dtype), n(rows, n_out).to(dtype)
        w2t, w1t = s["w2"].t().contiguous(), s["w1"].t().contiguous()
        e = lambda w: torch.empty(rows, w, device="cuda", dtype=dtype)
        make = lambda: dict(a=e(hidden), z=e(n_out), duv=e(2 * hidden), dx=e(n_in),
                            ku=buf(rows, hidden), kv=buf(rows, hidden), ka=buf(rows, hidden))

        def step(o):
            L.lrcnn_gated_ffn_forward(L.ACT_SILU, x, s["w1"], o["a"], s["b1"], s["w2"], s["b2"],
                                      o["z"], ckpt_u=o["ku"], ckpt_v=o["kv"])
            L.lrcnn_gated_ffn_backward(L.ACT_SILU, dz, w2t, o["duv"], ckpt_u=o["ku"],
                                       ckpt_v=o["kv"], ckpt_a=o["ka"], w1t=w1t, dx=o["dx"])
        got, want = make(), make()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(got)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(got)
        for i in range(3):
            x.mul_(1.125)
            for k in ("a", "z", "duv", "dx"):
                got[k].fill_(math.nan)
            graph.replay()
            step(want)
            torch.cuda.synchronize()
            for k in ("a", "z", "duv", "dx"):
                assert torch.equal(got[k], want[k]), (rows, i, k)
            for k in ("ku", "kv", "ka"):
                assert torch.equal(held(got[k], rows, hidden), held(want[k], rows, hidden)), k
