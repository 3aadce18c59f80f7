"""The feed-forward block with 8-bit checkpoints, all its operators together: its
output against float64, its gradients against the formulas on what its
checkpoints hold (tight) and against exact gradients (the 8 bits' error), and
a few training steps of trunk, block and head.

Tolerances (norm of the error over norm of the result). float32 on held
values: products over up to 192 features and sums over 96 rows, some 1e-6
each, four of them in a row: 2e-5. bfloat16: four or five roundings of 2^-9 on the
way: 2e-2. Against exact gradients: a step of 2^-6 of a group's largest value
in uniform error is 2^-6 / sqrt(12) = 0.5% of it, about 1% of the values' rms,
two or three of them on a path: 5e-2."""
import numpy as np
import pytest
import torch

from paper_2401_11471_amd import ffn
from paper_2401_11471_amd import lrcnn as L

pytestmark = pytest.mark.gpu


def rel(a, r):
    return float((a.double() - r).norm() / r.norm())


def act(u, kind):
    F = torch.nn.functional
    return {L.ACT_GELU: F.gelu, L.ACT_SILU: F.silu, L.ACT_RELU: F.relu}[kind](u)


def unpacked(ckpt, rows, cols):
    y = torch.empty(rows, cols, device="cuda")
    L.lrcnn_act8_unpack(ckpt, y)
    return y.double()


@pytest.mark.parametrize("dtype", [L.F32, L.BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("kind,gated", [(L.ACT_GELU, False), (L.ACT_SILU, True)],
                         ids=["gelu", "silu_gated"])
@pytest.mark.parametrize("rows,cols,hidden", [(96, 64, 192), (77, 40, 72)])
def test_block(rows, cols, hidden, kind, gated, dtype):
    print(f"block {rows} {cols} {hidden} {kind} {gated} {dtype}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(rows)
    tdt = torch.bfloat16 if dtype == L.BF16 else torch.float32

    def n(*s):
        return torch.randn(*s, generator=g, device="cuda")
    b = ffn.FeedForward(rows, cols, hidden, dtype, kind, gated, seed=3)
    for t in (b.norm1.gamma, b.norm2.gamma):
        t.add_(0.2 * n(cols))
    for t in (b.norm1.beta, b.norm2.beta, b.lin1.b, b.lin2.b):
        t.copy_(0.3 * n(t.numel()))
    x, dy = n(rows, cols).to(tdt), n(rows, cols).to(tdt)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    b.forward(x, y)
    b.backward(dy, dx)
    torch.cuda.synchronize()

    # exact, with float64 autograd
    leaf = lambda t: t.double().requires_grad_()
    X, W1, W2 = leaf(x), leaf(b.lin1.w), leaf(b.lin2.w)
    B1, B2, G1, G2, E1, E2 = (leaf(t) for t in (b.lin1.b, b.lin2.b, b.norm1.gamma, b.norm2.gamma,
                                                b.norm1.beta, b.norm2.beta))
    ln = lambda t, ga, be: torch.nn.functional.layer_norm(t, (cols,), ga, be, ffn.EPS)
    U = ln(X, G1, E1) @ W1.t() + B1
    A = act(U[:, :hidden], kind) * U[:, hidden:] if gated else act(U, kind)
    Y = ln(X + A @ W2.t() + B2, G2, E2)
    Y.backward(dy.double())
    fine = 2e-2 if dtype == L.BF16 else 2e-5
    assert rel(y, Y.detach()) < fine
    got = [(dx, X), (b.lin1.dw, W1), (b.lin2.dw, W2), (b.lin1.db, B1), (b.lin2.db, B2),
           (b.norm1.dgamma, G1), (b.norm2.dgamma, G2), (b.norm1.dbeta, E1), (b.norm2.dbeta, E2)]
    for i, (t, ref) in enumerate(got):
        assert rel(t, ref.grad) < 5e-2, i

    # the same chain on what the checkpoints hold
    def norm_back(dy, xh, rstd, ga, dres=0):
        q = dy * ga
        return rstd[:, None] * (q - q.mean(1, True) - xh * (q * xh).mean(1, True)) + dres
    with torch.no_grad():
        d = dy.double()
        xh1, xh2 = unpacked(b.norm1.ckpt, rows, cols), unpacked(b.norm2.ckpt, rows, cols)
        dt = norm_back(d, xh2, b.norm2.rstd.double(), G2)
        da = dt @ W2
    u = unpacked(b.k_u, rows, hidden).requires_grad_()
    v = unpacked(b.k_v, rows, hidden).requires_grad_() if gated else None
    a = act(u, kind) * v if gated else act(u, kind)
    a.backward(da)
    with torch.no_grad():
        du = torch.cat([u.grad, v.grad], 1) if gated else u.grad
        dh = du @ W1
        ref = {"dx": norm_back(dh, xh1, b.norm1.rstd.double(), G1, dt),
               "dw1": du.t() @ (xh1 * G1 + E1), "db1": du.sum(0), "db2": dt.sum(0),
               "dw2": dt.t() @ unpacked(b.k_a, rows, hidden), "dgamma1": (dh * xh1).sum(0),
               "dgamma2": (d * xh2).sum(0)}
    out = {"dx": dx, "dw1": b.lin1.dw, "db1": b.lin1.db, "db2": b.lin2.db, "dw2": b.lin2.dw,
           "dgamma1": b.norm1.dgamma, "dgamma2": b.norm2.dgamma}
    for k, r in ref.items():
        assert rel(out[k], r) < fine, k


def test_saved_bytes():
    b = ffn.FeedForward(1000, 64, 256)
    assert b.saved_bytes() < 1.05 * 1000 * (2 * 64 + 256) + 8 * 1000 + 4096


def test_training(capsys):
    ffn.main()
    losses = [float(l.split()[-1]) for l in capsys.readouterr().out.splitlines() if "loss" in l]
    assert np.isfinite(losses).all() and losses[-1] < 0.5 * losses[0]


@pytest.mark.parametrize("gated", [False, True], ids=["gelu", "silu_gated"])
def test_blocks_in_one_scratch(gated):
    """Three blocks in a row, the last one narrower, forward and then backward in
    the scratch of the first: the same bits as with a scratch each."""
    print(f"blocks in one scratch {gated}", flush=True)
    rows, cols, kind = 150, 64, L.ACT_SILU if gated else L.ACT_GELU
    g = torch.Generator(device="cuda").manual_seed(8)
    x0, d0 = (torch.randn(rows, cols, generator=g, device="cuda").bfloat16() for _ in range(2))

    def run(shared):
        blocks = []
        for i, hidden in enumerate((200, 200, 72)):
            scratch = blocks[0].scratch if shared and blocks else None
            blocks.append(ffn.FeedForward(rows, cols, hidden, L.BF16, kind, gated, seed=i,
                                          scratch=scratch))
        x, d = [x0], [d0]
        for b in blocks:
            x.append(torch.empty_like(x0))
            b.forward(x[-2], x[-1])
        for b in reversed(blocks):
            d.append(torch.empty_like(x0))
            b.backward(d[-2], d[-1])
        torch.cuda.synchronize()
        return x + d + [t for b in blocks for t in (b.lin1.dw, b.lin2.dw, b.lin1.db, b.lin2.db,
                                                    b.norm1.dgamma, b.norm2.dbeta)]
    own, shared = run(False), run(True)
    assert all(torch.isfinite(t).all() for t in own)
    assert all(torch.equal(p, q) for p, q in zip(own, shared))


@pytest.mark.parametrize("dtype", [L.F32, L.BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("gated", [False, True], ids=["gelu", "silu_gated"])
def test_update(gated, dtype):
    """update(lr) moves every parameter by -lr times its gradient: one rounding to
    the storage type, 2^-8 or 2^-23 of the value, and float32's product before it.
    The pass after it gives the bits of a new block with those parameters, so nothing
    of the old ones is left, the transposed weights among them."""
    print(f"update {gated} {dtype}", flush=True)
    rows, cols, hidden, lr, kind = 90, 48, 104, 0.25, L.ACT_SILU if gated else L.ACT_GELU
    tdt = torch.bfloat16 if dtype == L.BF16 else torch.float32
    g = torch.Generator(device="cuda").manual_seed(6)
    x, dy = (torch.randn(rows, cols, generator=g, device="cuda").to(tdt) for _ in range(2))

    def params(b):
        return [b.lin1.w, b.lin2.w, b.lin1.b, b.lin2.b, b.norm1.gamma, b.norm2.gamma, b.norm1.beta,
                b.norm2.beta]

    def grads(b):
        return [b.lin1.dw, b.lin2.dw, b.lin1.db, b.lin2.db, b.norm1.dgamma, b.norm2.dgamma,
                b.norm1.dbeta, b.norm2.dbeta]

    def step(b):
        y, dx = torch.empty_like(x), torch.empty_like(x)
        b.forward(x, y)
        b.backward(dy, dx)
        torch.cuda.synchronize()
        return [y, dx] + [t.clone() for t in grads(b)]
    b = ffn.FeedForward(rows, cols, hidden, dtype, kind, gated, seed=1)
    first = step(b)
    old, d = [t.clone() for t in params(b)], first[2:]
    b.update(lr)
    for i, (new, was, grad) in enumerate(zip(params(b), old, d)):
        want = was.double() - lr * grad.double()
        ulp = 2.0 ** -8 if new.dtype is torch.bfloat16 else 2.0 ** -23
        assert (new.double() - want).abs().le(ulp * want.abs() + 2.0 ** -23 * was.double().abs()
                                              + 1e-37).all(), i
        assert (new != was).float().mean() > 0.5, i
    for lin in (b.lin1, b.lin2):
        assert torch.equal(lin.wt, lin.w.t())
    fresh = ffn.FeedForward(rows, cols, hidden, dtype, kind, gated, seed=2)
    for t, s in zip(params(fresh), params(b)):
        t.copy_(s)
    for lin in (fresh.lin1, fresh.lin2):
        lin.wt.copy_(lin.w.t())
    got, want = step(b), step(fresh)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    # (norm2's dbeta, the sum of dy, is the one result without a parameter in it)
    assert torch.equal(got[-1], first[-1])
    assert not any(torch.equal(p, q) for p, q in zip(got[:-1], first))
