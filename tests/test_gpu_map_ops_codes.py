"""The group norm's checkpoint, exponents and codes: a group's exponent is that of its largest
magnitude, neither side of it but where the map's own error reaches the other. The error
of xh, and what it is made of, is that of the group norm's other tests."""
import numpy as np
import pytest
import torch

from oracle import block as OB
from oracle import map_ops as OM
from paper_2401_11471_amd import lrcnn as L
from test_gpu_map_ops import SIZES, TYPES, buf, features, matrix, np64, t_error, workspace

pytestmark = pytest.mark.gpu


@TYPES
@SIZES
def test_group_norm_codes(batch, pixels, cols, groups, dtype):
    print("group norm codes", batch, pixels, cols, groups, dtype, flush=True)
    rng = np.random.default_rng(pixels + 7 * cols)
    rows = batch * pixels
    x = matrix(features(rng, rows, cols), dtype)
    y, ck = torch.empty_like(x), buf(L.lrcnn_act8_bytes(rows, cols))
    L.lrcnn_group_norm_forward(L.ACT_NONE, x, None, None, 1e-3, y, batch, groups,
                               workspace(batch, pixels, cols, groups), ckpt=ck)
    one, zero = np.ones(cols), np.zeros(cols)
    X = np64(x)
    _, _, xh, _, rstd = OM.group_norm(X, batch, groups, 1.0, 0.0, np.float64(np.float32(1e-3)), "none")
    err = t_error(X, xh, xh, rstd, batch, groups, one, zero)
    q, e = OB.unpack_bytes(ck.cpu().numpy(), rows, cols)
    wrong_groups, wrong = OB.misfits(q, e, xh, err)
    assert not wrong_groups.any() and not wrong.any()
    assert (q[:, cols:] == 0).all()
    # Next to no group is so near a power of two that two exponents could be right. (Counted
    # without the rows of zeros: they all hold -mean rstd of their group of channels, so an
    # image where that is near one has a seventh of its rows there, 1.1% of 40 images' groups.)
    low, high = OB.encode(np.maximum(np.abs(xh) - err, 0))[1], OB.encode(np.abs(xh) + err)[1]
    assert (low != high)[np.abs(X).max(1) > 0].mean() < 0.01 or rows * cols < 1000
