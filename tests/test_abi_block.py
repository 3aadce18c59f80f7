"""Refusals of the feed-forward block entry points and of their binding, and
their size queries: host code only. Nothing is enqueued by a refused call."""
import ctypes as C

import pytest
import torch

from paper_2401_11471_amd import lrcnn as L

P = 1 << 20  # a pointer that is never followed
EINVAL, ESHAPE, EWORKSPACE, EDTYPE = -1, -2, -4, -6


def last():
    return L.LIB.lrcnn_last_error().decode()


def test_checkpoint_bytes():
    for rows, cols in [(0, 1), (1, 1), (1, 32), (5, 33), (67800, 2048)]:
        pitch = -(-cols // 32) * 32
        a = lambda n: -(-n // 256) * 256
        assert L.lrcnn_act8_bytes(rows, cols) == a(rows * pitch) + a(rows * pitch // 32)
    for rows, cols in [(-1, 4), (1, 0), (1, -3), (1 << 41, 1), (1, 1 << 31), (1 << 30, 1 << 30)]:
        with pytest.raises(L.LrcnnError) as e:
            L.lrcnn_act8_bytes(rows, cols)
        assert e.value.code == ESHAPE
    assert L.LIB.lrcnn_act8_bytes(1, 1, None) == EINVAL


def test_pack_and_unpack_refuse():
    pack, unpack = L.LIB.lrcnn_act8_pack, L.LIB.lrcnn_act8_unpack
    assert pack(2, 8, 7, P, 0, P, None) == EDTYPE
    assert pack(2, 8, L.F32, None, 0, P, None) == EINVAL and "x is null" in last()
    assert pack(2, 8, L.F32, P, 0, None, None) == EINVAL
    assert pack(2, 8, L.F32, P + 2, 0, P, None) == EINVAL and "misaligned" in last()
    assert pack(2, 8, L.BF16, P + 1, 0, P, None) == EINVAL
    assert pack(2, 8, L.F32, P, 0, P + 8, None) == EINVAL
    assert pack(2, 8, L.F32, P, 7, P, None) == ESHAPE
    assert pack(2, 8, L.F32, P, -8, P, None) == ESHAPE
    assert unpack(2, 8, L.F32, P, None, 0, None) == EINVAL
    assert unpack(2, 8, L.F32, None, P, 0, None) == EINVAL
    assert unpack(2, 0, L.F32, P, P, 0, None) == ESHAPE
    # no rows: nothing to do, nothing to check
    assert pack(0, 8, L.F32, None, 0, None, None) == 0
    assert unpack(0, 8, L.BF16, None, None, 0, None) == 0


def ln_fwd(rows=2, cols=8, dtype=L.F32, x=P, ldx=0, res=None, gamma=P, beta=P, eps=1e-5,
           total=None, y=P, mean=P, rstd=P, ckpt=None):
    return L.LIB.lrcnn_layer_norm_forward(rows, cols, dtype, x, ldx, res, 0, gamma, beta, eps,
                                          total, 0, y, 0, mean, rstd, ckpt, None)


def test_layer_norm_forward_refuses():
    assert ln_fwd(dtype=5) == EDTYPE
    assert ln_fwd(rows=-1) == ESHAPE
    assert ln_fwd(cols=16385) == ESHAPE and "16384" in last()
    assert ln_fwd(x=None) == EINVAL
    assert ln_fwd(y=None) == EINVAL
    assert ln_fwd(x=P + 2) == EINVAL
    assert ln_fwd(ldx=4) == ESHAPE
    assert ln_fwd(total=P) == EINVAL and "residual" in last()
    assert ln_fwd(gamma=P + 2) == EINVAL
    assert ln_fwd(rstd=P + 1) == EINVAL
    assert ln_fwd(ckpt=P + 4) == EINVAL
    for eps in (-1e-5, float("nan"), float("inf")):
        assert ln_fwd(eps=eps) == EINVAL
    assert ln_fwd(rows=0, x=None, y=None) == 0


def ln_bwd(rows=2, cols=8, dtype=L.F32, dy=P, x=P, mean=P, ckpt=None, rstd=P, gamma=P, dx=P,
           dgamma=P, dbeta=P, ws=P, ws_bytes=1 << 30):
    return L.LIB.lrcnn_layer_norm_backward(rows, cols, dtype, dy, 0, x, 0, mean, ckpt, rstd,
                                           gamma, None, 0, dx, 0, dgamma, dbeta, 0, ws, ws_bytes,
                                           None)


def test_layer_norm_backward_refuses():
    assert ln_bwd(dtype=2) == EDTYPE
    assert ln_bwd(cols=0) == ESHAPE
    assert ln_bwd(dy=None) == EINVAL
    assert ln_bwd(dx=None) == EINVAL
    assert ln_bwd(rstd=None) == EINVAL
    assert ln_bwd(x=None, mean=None) == EINVAL        # neither x nor ckpt
    assert ln_bwd(ckpt=P) == EINVAL                    # both
    assert ln_bwd(mean=None) == EINVAL                 # x without mean
    assert ln_bwd(x=None, ckpt=P) == EINVAL            # mean without x
    assert ln_bwd(ws=None) == EINVAL
    assert ln_bwd(ws=P + 8) == EINVAL
    need = L.lrcnn_layer_norm_workspace_bytes(2, 8)
    assert ln_bwd(ws_bytes=need - 1) == EWORKSPACE and str(need) in last()
    assert ln_bwd(dgamma=P + 2) == EINVAL
    with pytest.raises(L.LrcnnError) as e:
        L.lrcnn_layer_norm_workspace_bytes(4, 16385)
    assert e.value.code == ESHAPE


def act_fwd(kind=L.ACT_SILU, rows=2, cols=8, dtype=L.F32, u=P, v=None, a=P, ku=None, kv=None,
            ka=None, ldu=0):
    return L.LIB.lrcnn_activation_forward(rows, cols, dtype, kind, u, ldu, v, 0, a, 0, ku, kv, ka,
                                          None)


def act_bwd(kind=L.ACT_SILU, rows=2, cols=8, dtype=L.F32, da=P, u=P, v=None, ku=None, kv=None,
            du=P, dv=None, ka=None):
    return L.LIB.lrcnn_activation_backward(rows, cols, dtype, kind, da, 0, u, 0, v, 0, ku, kv, du,
                                           0, dv, 0, ka, None)


def test_activations_refuse():
    for kind in (-1, 4):
        assert act_fwd(kind=kind) == EINVAL
        assert act_bwd(kind=kind) == EINVAL
    assert act_fwd(dtype=9) == EDTYPE
    assert act_fwd(u=None) == EINVAL
    assert act_fwd(a=None) == EINVAL and "no output" in last()
    assert act_fwd(kv=P) == EINVAL
    assert act_fwd(ldu=7) == ESHAPE
    assert act_fwd(ka=P + 1) == EINVAL
    assert act_bwd(da=None) == EINVAL
    assert act_bwd(du=None) == EINVAL
    assert act_bwd(u=None) == EINVAL
    assert act_bwd(ku=P) == EINVAL                     # u twice
    assert act_bwd(v=P) == EINVAL                      # gated without dv
    assert act_bwd(dv=P) == EINVAL                     # dv without v
    assert act_bwd(u=None, ku=P, v=P, dv=P) == EINVAL  # v full-width, u not
    assert act_bwd(kv=P, dv=P) == EINVAL
    assert act_bwd(ka=P + 8) == EINVAL
    assert act_fwd(rows=0, u=None) == 0 and act_bwd(rows=0, da=None) == 0


def wgrad(rows=4096, n_in=64, n_out=64, dtype=L.F32, dy=P, lddy=0, ckpt=P, scale=None, shift=None,
          dw=P, db=P, ws=P, ws_bytes=1 << 40):
    return L.LIB.lrcnn_linear_wgrad(rows, n_in, n_out, dtype, dy, lddy, ckpt, scale, shift, dw, db,
                                    0, ws, ws_bytes, None)


def test_linear_wgrad_refuses():
    assert wgrad(dtype=3) == EDTYPE
    assert wgrad(n_in=0) == ESHAPE
    assert wgrad(n_out=0) == ESHAPE
    assert wgrad(rows=-1) == ESHAPE
    assert wgrad(dy=None) == EINVAL
    assert wgrad(dy=P + 2) == EINVAL
    assert wgrad(lddy=63) == ESHAPE
    assert wgrad(ckpt=None) == EINVAL
    assert wgrad(ckpt=P + 8) == EINVAL
    assert wgrad(dw=None) == EINVAL
    assert wgrad(scale=P + 1) == EINVAL
    need = L.lrcnn_linear_wgrad_workspace_bytes(4096, 64, 64)
    assert need > 0
    assert wgrad(ws=None) == EINVAL
    assert wgrad(ws_bytes=need - 1) == EWORKSPACE


def test_binding_refuses_tensors_that_do_not_agree():
    f = lambda *s, **k: torch.zeros(*s, **k)
    x, ck = f(4, 40), f(L.lrcnn_act8_bytes(4, 40), dtype=torch.uint8)

    def refused(code, fn, *a, **k):
        with pytest.raises(L.LrcnnError) as e:
            fn(*a, stream=0, **k)
        assert e.value.code == code, e.value

    refused(EINVAL, L.lrcnn_act8_pack, f(4, 4, 4), ck)
    refused(EDTYPE, L.lrcnn_act8_pack, x.half(), ck)
    refused(EINVAL, L.lrcnn_act8_pack, x, ck[:-1])
    refused(EINVAL, L.lrcnn_act8_pack, x, ck.float())
    refused(EINVAL, L.lrcnn_act8_pack, f(40, 4).t(), ck)       # columns apart
    refused(EINVAL, L.lrcnn_act8_pack, f(1, 40).expand(4, 40), ck)  # rows overlap
    refused(EINVAL, L.lrcnn_act8_unpack, ck, f(8, 40))
    refused(EINVAL, L.lrcnn_layer_norm_forward, x, f(40), f(39), 1e-5, f(4, 40))
    refused(EINVAL, L.lrcnn_layer_norm_forward, x, f(40), f(40), 1e-5, f(4, 41))
    refused(EINVAL, L.lrcnn_layer_norm_forward, x, f(40), f(40), 1e-5, f(4, 40), rstd=f(5))
    refused(EINVAL, L.lrcnn_layer_norm_forward, x, f(40), f(40), 1e-5, f(4, 40),
            residual=f(4, 40).bfloat16())
    refused(EINVAL, L.lrcnn_layer_norm_backward, x, f(4), f(40), f(4, 40), f(41), None,
            f(1 << 16, dtype=torch.uint8), x=x, mean=f(4))
    refused(EWORKSPACE, L.lrcnn_layer_norm_backward, x, f(4), f(40), f(4, 40), f(40), None,
            f(16, dtype=torch.uint8), x=x, mean=f(4))
    refused(EINVAL, L.lrcnn_activation_forward, L.ACT_GELU, x, f(4, 40), v=f(4, 39))
    refused(EINVAL, L.lrcnn_activation_backward, L.ACT_GELU, x, f(4, 40), u=f(3, 40))
    refused(EINVAL, L.lrcnn_linear_wgrad, x, ck, f(39, 40))
    refused(EINVAL, L.lrcnn_linear_wgrad, x, ck, f(40, 80))
    refused(EINVAL, L.lrcnn_linear_wgrad, x, ck, f(40, 40).double())
    refused(EINVAL, L.lrcnn_linear_wgrad, x, ck, f(40, 40), scale=f(41))


# name, and a call of host tensors that agree with each other
CALLS = {
    "lrcnn_act8_pack": lambda f, b, **k: L.lrcnn_act8_pack(f(4, 40), b, **k),
    "lrcnn_act8_unpack": lambda f, b, **k: L.lrcnn_act8_unpack(b, f(4, 40), **k),
    "lrcnn_layer_norm_forward": lambda f, b, **k: L.lrcnn_layer_norm_forward(
        f(4, 40), f(40), f(40), 1e-5, f(4, 40), rstd=f(4), ckpt=b, **k),
    "lrcnn_layer_norm_backward": lambda f, b, **k: L.lrcnn_layer_norm_backward(
        f(4, 40), f(4), f(40), f(4, 40), f(40), f(40), b, ckpt=b, **k),
    "lrcnn_activation_forward": lambda f, b, **k: L.lrcnn_activation_forward(
        L.ACT_SILU, f(4, 40), f(4, 40), v=f(4, 40), ckpt_u=b, **k),
    "lrcnn_activation_backward": lambda f, b, **k: L.lrcnn_activation_backward(
        L.ACT_GELU, f(4, 40), f(4, 40), ckpt_u=b, **k),
    "lrcnn_linear_wgrad": lambda f, b, **k: L.lrcnn_linear_wgrad(
        f(4, 10), b, f(10, 40), b, db=f(10), **k),
}


@pytest.mark.parametrize("name", list(CALLS))
@pytest.mark.parametrize("stream", [{}, {"stream": 0}], ids=["current", "given"])
def test_binding_refuses_host_tensors(name, stream, monkeypatch):
    """Host memory never reaches the library, whose kernels would follow its pointers."""
    reached = []
    monkeypatch.setattr(L.LIB, name, lambda *a: reached.append(a) or 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 0, raising=False)
    with pytest.raises(L.LrcnnError) as e:
        CALLS[name](torch.zeros, torch.zeros(1 << 16, dtype=torch.uint8), **stream)
    assert e.value.code == EINVAL and "GPU" in str(e.value)
    assert not reached


@pytest.mark.parametrize("stream", [None, 0, 77])
def test_binding_refuses_tensors_of_another_gpu(stream, monkeypatch):
    """Tensors of GPU 1 are worked on while it is current, in its stream, and refused
    while GPU 0 is: the library launches on the current device."""
    calls = []
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 100 + dev, raising=False)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 1)
    for name, call in CALLS.items():
        monkeypatch.setattr(L.LIB, name, lambda *a: calls.append(a[-1]) or 0)
        run = lambda: call(torch.zeros, torch.zeros(1 << 16, dtype=torch.uint8), stream=stream)
        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
        with pytest.raises(L.LrcnnError) as e:
            run()
        assert e.value.code == EINVAL and "cuda:1" in str(e.value) and not calls
        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)
        run()
        assert calls.pop() == (101 if stream is None else stream) and not calls


@pytest.mark.parametrize("n_in,n_out,dtype,last", [
    (2048, 2048, L.BF16, 67800), (512, 512, L.BF16, 6400), (256, 173, L.BF16, 540000),
    (64, 64, L.F32, 16000), (512, 2048, L.F32, 4000), (2048, 8192, L.BF16, 67800),
    (515, 300, L.F32, 30000), (33, 7, L.BF16, 30000), (300, 3000, L.BF16, 9000)])
def test_linear_wgrad_workspace_serves_fewer_rows(n_in, n_out, dtype, last):
    """The workspace of the largest band or micro-batch is enough for all: it never
    shrinks as the rows grow, and stays within what two (128 x 128) or one
    (256 x 256) float32 tiles a CU take."""
    need = [L.lrcnn_linear_wgrad_workspace_bytes(r, n_in, n_out, dtype)
            for r in range(0, last, max(1, last // 3000))]
    assert need == sorted(need)
    assert need[0] == 0 and need[-1] <= 256 * 256 * 256 * 4 + 256 * n_out * 4 + 512


def test_linear_wgrad_takes_the_workspace_it_asks_for():
    """A split weight gradient refuses anything less, also where a call of these
    rows alone would fit."""
    for rows in range(32 * 100, 32 * 200, 37):
        need = L.lrcnn_linear_wgrad_workspace_bytes(rows, 64, 64)
        assert wgrad(rows=rows, ws_bytes=need - 1) == EWORKSPACE and str(need) in last()
