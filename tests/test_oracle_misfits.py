"""The oracle's test of a checkpoint: what it lets pass and what it does not."""
import numpy as np

from oracle import block as OB


def test_misfits():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((40, 75))
    x[7, :32] = 0
    x[8, 40] = 127.5 / 64                          # from here on the next step
    q, e = OB.encode(x)
    err = np.full(x.shape, 1e-6)
    clean = lambda *a: not any(m.any() for m in OB.misfits(*a))
    assert clean(q, e, x, err) and clean(q, e, x, 0.0)
    assert clean(*OB.encode(x + 0.9e-6), x, err)
    # a step twice as wide everywhere, its codes rounded anew: one bit of every code lost
    wide = e + 1
    step = np.repeat(np.exp2(wide.astype(float) - 133), 32, 1)
    pad = np.zeros(q.shape)
    pad[:, :75] = x
    groups, _ = OB.misfits(np.rint(pad / step).astype(np.int8), wide, x, err)
    assert groups.sum() >= groups.size - 1         # (but the one next to the threshold)
    groups, elements = OB.misfits(q, e - 1, x, err)
    assert groups[:7].all() and elements.any()
    # a code off by one, and a value past what it is known to
    bad = q.copy()
    bad[5, 50] += 1
    assert OB.misfits(bad, e, x, err)[1][5, 50]
    assert not clean(*OB.encode(x + 0.1), x, err)
