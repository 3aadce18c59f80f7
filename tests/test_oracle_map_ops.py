"""The oracle of group norm, dropout and the gated feed-forward block: its gradients
against differences, its generator against the published known answers."""
import numpy as np
import pytest

from oracle import map_ops as OM

KINDS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def difference(f, x, eps=1e-5):
    """Gradient of the scalar f by central differences."""
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        old = x[i]
        x[i] = old + eps
        hi = f()
        x[i] = old - eps
        lo = f()
        x[i] = old
        g[i] = (hi - lo) / (2 * eps)
    return g


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("batch,pixels,cols,groups", [(2, 3, 6, 2), (1, 4, 5, 1), (3, 2, 4, 4)])
def test_group_norm_gradients(batch, pixels, cols, groups, kind):
    rng = np.random.default_rng(batch * cols)
    x, dy = rng.standard_normal((2, batch * pixels, cols))
    gamma, beta = 1 + 0.3 * rng.standard_normal(cols), 0.3 * rng.standard_normal(cols)
    f = lambda: (OM.group_norm(x, batch, groups, gamma, beta, 1e-3, kind)[0] * dy).sum()
    _, t, xh, mean, rstd = OM.group_norm(x, batch, groups, gamma, beta, 1e-3, kind)
    assert np.abs(t).min() > 1e-3  # no kink within the differences' reach
    got = OM.group_norm_backward(dy, xh, rstd, batch, groups, gamma, beta, kind)
    for g, v in zip(got, (x, gamma, beta)):
        assert np.allclose(g, difference(f, v), rtol=1e-5, atol=1e-7)
    assert np.allclose(xh, (x - OM.spread(mean, pixels, cols)) * OM.spread(rstd, pixels, cols))


@pytest.mark.parametrize("kind", KINDS[1:])
def test_gated_gradients(kind):
    rng = np.random.default_rng(4)
    u, v, da = rng.standard_normal((3, 4, 3))
    x, w1, b1 = rng.standard_normal((4, 5)), rng.standard_normal((6, 5)), rng.standard_normal(6)
    u, v, a = OM.gated(x, w1, b1, kind)
    f = lambda: (OM.gated(x, w1, b1, kind)[2] * da).sum()
    duv = np.concatenate(OM.gated_backward(da, u, v, kind), 1)
    assert np.allclose(duv @ w1, difference(f, x), rtol=1e-5, atol=1e-7)
    assert np.allclose(duv.T @ x, difference(f, w1), rtol=1e-5, atol=1e-7)


@pytest.mark.parametrize("counter,key,words", [
    ((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
    ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
    ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0),
     (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))])
def test_philox_known_answers(counter, key, words):
    """The generator's published known answers (zeros, ones, digits of pi)."""
    assert tuple(int(w) for w in OM.philox4x32(counter, key)) == words


def test_dropout_bits():
    bits = OM.dropout_bits(-5, 2 ** 63, 300, 41)
    assert bits.shape == (300, 41) and bits.min() >= 0 and bits.max() < 65536
    # a band draws what the whole draws; other sites and offsets draw other bits
    assert np.array_equal(OM.dropout_bits(-5, 2 ** 63, 20, 41, first_row=280), bits[280:])
    for kw in (dict(site=1), dict(offset=1)):
        a = dict(dict(seed=-5, offset=2 ** 63, rows=300, cols=41), **kw)
        assert (OM.dropout_bits(**a) == bits).mean() < 0.01
    # mean and spread of uniform bits: 12300 of them, within five standard errors
    assert abs(bits.mean() - 32767.5) < 5 * 65536 / np.sqrt(12 * bits.size)
    x = np.full((300, 41), 3.0)
    y = OM.dropout(x, 0.25, bits)
    assert set(np.unique(y)) == {0.0, 4.0}
    assert abs((y == 0).mean() - 0.25) < 5 * np.sqrt(0.25 * 0.75 / bits.size)
    assert (OM.dropout(x, 1.0, bits) == 0).all() and (OM.dropout(x, 0.0, bits) == 3).all()
