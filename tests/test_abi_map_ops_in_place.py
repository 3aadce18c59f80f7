"""Outputs in place of an input with another row stride: their rows would be written over
others that are still to be read. Host code only, no kernel is reached by a refused call."""
from paper_2401_11471_amd import lrcnn as L

P, Q, R = (1 << 20, 1 << 21, 1 << 22)  # pointers that are never followed
EINVAL, ESHAPE = -1, -2


def last():
    return L.LIB.lrcnn_last_error().decode()


def refused(status, name):
    assert status == EINVAL
    assert name + " is an input's memory with another row stride" in last()


def ffn_bwd(uv, lduv, duv, ldduv, rows=2, w2t=R):
    return L.LIB.lrcnn_gated_ffn_backward(rows, 8, 16, 8, L.F32, L.ACT_SILU, P, 0, w2t, uv, lduv,
                                          None, None, duv, ldduv, None, None, None, 0, None)


def test_gated_ffn_backward_in_place_of_other_rows():
    refused(ffn_bwd(Q, 0, Q, 40), "duv")
    refused(ffn_bwd(Q, 40, Q, 0), "duv")
    refused(ffn_bwd(Q, 40, Q, 48), "duv")
    # a stride too small is still that; no rows, nothing to refuse
    assert ffn_bwd(Q, 0, Q, 31) == ESHAPE
    assert ffn_bwd(Q, 0, Q, 40, rows=0) == 0


def gn_fwd(x, ldx, y, ldy, batch=2, pixels=3):
    return L.LIB.lrcnn_group_norm_forward(batch, pixels, 8, 2, L.F32, L.ACT_SILU, x, ldx, None,
                                          None, 1e-5, y, ldy, None, None, None, P, 1 << 40, None)


def gn_bwd(dy, lddy, x, ldx, dx, lddx, batch=2, pixels=3, ckpt=None):
    return L.LIB.lrcnn_group_norm_backward(batch, pixels, 8, 2, L.F32, L.ACT_SILU, dy, lddy, x, ldx,
                                           P if x else None, ckpt, P, None, None, dx, lddx, None,
                                           None, 0, P, 1 << 40, None)


def test_group_norm_in_place_of_other_rows():
    for a, b in ((0, 16), (16, 0), (16, 24)):
        refused(gn_fwd(Q, a, Q, b), "y")
        refused(gn_bwd(Q, a, R, 0, Q, b), "dx")
        refused(gn_bwd(Q, a, None, 0, Q, b, ckpt=R), "dx")
        refused(gn_bwd(R, 0, Q, a, Q, b), "dx")
    refused(gn_fwd(Q, 0, Q, 16, batch=1, pixels=2), "y")
    assert gn_fwd(Q, 0, Q, 7) == ESHAPE and gn_bwd(Q, 0, R, 0, Q, 7) == ESHAPE


def drop(x, ldx, res, ldr, y, ldy, rows=2):
    return L.LIB.lrcnn_dropout(rows, 8, L.F32, x, ldx, res, ldr, 0.5, P, 0, 0, y, ldy, None)


def test_dropout_in_place_of_other_rows():
    for a, b in ((0, 16), (16, 0), (16, 24)):
        refused(drop(Q, a, None, 0, Q, b), "y")
        refused(drop(Q, a, R, 0, Q, b), "y")
        refused(drop(R, 0, Q, a, Q, b), "y")
    assert drop(Q, 0, None, 0, Q, 7) == ESHAPE
    assert drop(Q, 0, None, 0, Q, 16, rows=0) == 0
