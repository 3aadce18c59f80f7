"""The oracle of the feed-forward block operators against independent
statements: codes by scalar search over all 255 of them, bfloat16 exactness,
gradients against central differences and torch's float64 library routines."""
import math

import numpy as np
import pytest
import torch

from oracle import block as OB


def test_codes_are_nearest_and_steps_minimal():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((40, 70)) * np.exp(rng.uniform(-30, 30, (40, 1)))
    x[3] = 0
    q, e = OB.encode(x)
    assert q.shape == (40, 96) and e.shape == (40, 3)
    assert (q[:, 70:] == 0).all()
    for r in range(40):
        for g in range(3):
            seg = np.zeros(32)
            part = x[r, 32 * g:32 * g + 32]
            seg[:len(part)] = part
            step = 2.0 ** (int(e[r, g]) - 133)
            codes = q[r, 32 * g:32 * g + 32].astype(float)
            # nearest: no other code is nearer
            assert (np.abs(seg - codes * step) <= 0.5 * step).all()
            assert np.abs(codes).max() <= 127
            # half the step would not hold the largest value (unless at the floor)
            if e[r, g] > 7:
                assert np.rint(np.abs(seg).max() / (step / 2)) > 127


def test_code_edges():
    # rounds to 128 steps of 2^-6: the next step; just below: not
    top = 2.0 - 2.0 ** -7
    for v, want_e, want_q in [(top, 128, 64), (np.nextafter(top, 0), 127, 127), (1.0, 127, 64),
                              (0.0, 7, 0), (2.0 ** -126, 7, 1), (2.0 ** -140, 7, 0),
                              (3.3895313892515355e38, 254, 127), (-3.4e38, 254, -127)]:
        q, e = OB.encode(np.array([[v]]))
        assert (e[0, 0], q[0, 0]) == (want_e, want_q), v
    for v in (math.inf, -math.inf, math.nan):
        q, e = OB.encode(np.array([[1.0, v]]))
        assert e[0, 0] == 255 and (q == 0).all()
        assert np.isnan(OB.decode(q, e, 2)).all()
    # ties go to even codes
    q, _ = OB.encode(np.array([[64.0, 2.5, 3.5, -2.5, -3.5]]))
    assert list(q[0, 1:5]) == [2, 4, -2, -4]


def test_values_are_exact_in_bfloat16():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((64, 100)) * np.exp(rng.uniform(-80, 80, (64, 1)))
    v = OB.held(x)
    t = torch.from_numpy(v)
    assert torch.equal(t.bfloat16().double(), t)
    assert np.array_equal(OB.held(v), v)  # packing what is held changes nothing


def test_buffer_layout():
    rng = np.random.default_rng(2)
    q, e = OB.encode(rng.standard_normal((5, 70)))
    buf = OB.pack_bytes(q, e)
    assert len(buf) == 512 + 256
    q2, e2 = OB.unpack_bytes(buf, 5, 70)
    assert np.array_equal(q, q2) and np.array_equal(e, e2)


def _central(f, x, d, h=1e-6):
    return (f(x + h * d) - f(x - h * d)) / (2 * h)


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 2), (5, 33), (7, 64)])
def test_layer_norm_gradient(rows, cols):
    rng = np.random.default_rng(rows * cols)
    x, dy = rng.standard_normal((2, rows, cols))
    ga, be = 1 + 0.3 * rng.standard_normal(cols), rng.standard_normal(cols)
    eps = 1e-3

    def loss(x, ga, be):
        return (OB.layer_norm(x, ga, be, eps)[0] * dy).sum()
    _, xh, _, rstd = OB.layer_norm(x, ga, be, eps)
    dx, dg, db = OB.layer_norm_backward(dy, xh, rstd, ga)
    d = rng.standard_normal((rows, cols))
    assert (dx * d).sum() == pytest.approx(_central(lambda t: loss(t, ga, be), x, d), abs=1e-6)
    d = rng.standard_normal(cols)
    assert (dg * d).sum() == pytest.approx(_central(lambda t: loss(x, t, be), ga, d), abs=1e-6)
    assert (db * d).sum() == pytest.approx(_central(lambda t: loss(x, ga, t), be, d), abs=1e-6)
    y = torch.nn.functional.layer_norm(torch.from_numpy(x), (cols,), torch.from_numpy(ga),
                                       torch.from_numpy(be), eps)
    assert np.allclose(OB.layer_norm(x, ga, be, eps)[0], y.numpy(), atol=1e-12)


@pytest.mark.parametrize("kind", ["relu", "gelu", "gelu_tanh", "silu"])
def test_activation_gradient(kind):
    u = np.concatenate([np.linspace(-9, 9, 400) + 1e-3, [0.0]])
    f, df = OB.activation(u, kind)
    diff = _central(lambda t: OB.activation(t, kind)[0], u[:-1], np.ones(400))
    assert np.allclose(df[:-1], diff, atol=1e-8)
    t = torch.from_numpy(u)
    F = torch.nn.functional
    want = {"relu": F.relu(t), "gelu": F.gelu(t), "gelu_tanh": F.gelu(t, approximate="tanh"),
            "silu": F.silu(t)}[kind]
    assert np.allclose(f, want.numpy(), atol=1e-12)


def test_linear_wgrad_gradient():
    rng = np.random.default_rng(5)
    dy, q = rng.standard_normal((9, 4)), rng.standard_normal((9, 6))
    sc, sh = rng.standard_normal((2, 6))
    w, b = rng.standard_normal((4, 6)), rng.standard_normal(4)
    dw, db = OB.linear_wgrad(dy, q, sc, sh)
    d = rng.standard_normal((4, 6))
    assert (dw * d).sum() == pytest.approx(
        _central(lambda t: (((q * sc + sh) @ t.T + b) * dy).sum(), w, d), abs=1e-7)
    assert np.allclose(db, dy.sum(0))
