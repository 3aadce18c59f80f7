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
