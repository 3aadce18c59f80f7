"""A feed-forward block behind a convolution trunk, trained with its saved
activations in 8 bits.

The block works on the rows (pixels) of a feature map x [rows][cols]:

    h = norm1(x),  u = h W1^T + b1,  a = f(u)   (gated: f(u) * v, u and v the
    halves of one product),  z = a W2^T + b2,  y = norm2(x + z)

Between forward and backward it keeps, per row, an 8-bit checkpoint of norm1's
normalised row (for norm1's backward pass and, with its scale and shift, for W1's
gradient), of u (and v) and of norm2's normalised row, and two float32
statistics: cols * 2 + hidden bytes (twice hidden if gated) and a 32nd, where
bfloat16 copies of what the backward pass reads (x, h, x + z, u, a and, gated, v)
take about three times that. a is formed again from u. What a pass
uses at full width is scratch that blocks share (``scratch=``), so each block
after the first adds only what it keeps.

The passes and the update of the weights run in the HIP library, the linear
products and input gradients as 1x1 convolutions; the biases' and norms'
updates and the weights' transposes are torch operations.

``fused``: a gated block's products run as two kernels a pass, the activation in the
first one's registers: u and v then never exist at full width, and a is formed from their
float32 values. Forward + backward pass in us, separate kernels and fused:

====================  =======  ==============  =============
block                 storage  separate        fused
====================  =======  ==============  =============
67800 x 2048 x 8192   bf16     13540 + 19680   5700 + 12780
3136 x 1024 x 2736    bf16     156 + 262       91 + 214
392 x 512 x 2048      float32  64 + 114        58 + 114
256 x 2048 x 8192     bf16     83 + 189        64 + 220
33 x 2048 x 8192      bf16     48 + 139        52 + 186
1 x 2048 x 8192       bf16     43 + 129        34 + 114
====================  =======  ==============  =============

So fused is the choice from some 300 rows on and for a few; from 17 to some 300 rows of a
wide block it is not where the block is trained: dx there has few tiles and a long depth,
which fused products do not split over workgroups. The default is separate. ``dropout``: y = norm2(x + dropout(z)), whose mask is drawn again in the
backward pass from the generator's state in device memory. ``GroupNorm`` normalises and
activates the trunk's map in front of the block.

``python -m paper_2401_11471_amd.ffn`` trains a small trunk, block and classifier
head on random labelled images; with ``--fused`` the trunk's map is group-normalised, the
block is fused and drops out a tenth.
"""
from __future__ import annotations

import math

import torch

from . import lrcnn as L
from .device import torch_dtype

EPS = 1e-5


class Linear:
    """y = x W^T + b on [rows][n_in] as a 1x1 convolution with an affine of scale 1
    and shift b; its input gradient as one with W transposed."""

    def __init__(self, rows, n_in, n_out, dtype, device, generator):
        self.rows, self.n_in, self.n_out, self.dtype = rows, n_in, n_out, dtype
        tdt = torch_dtype(dtype)

        def f32(*shape, value=0.0):
            return torch.full(shape, value, device=device)
        w = torch.randn(n_out, n_in, generator=generator) / math.sqrt(n_in)
        self.w = w.to(device=device, dtype=tdt)
        self.wt = self.w.t().contiguous()
        self.b, self.one = f32(n_out), f32(n_out, value=1.0)
        self.dw, self.db = f32(n_out, n_in), f32(n_out)

        def plan(c_in, c_out, affine):
            nodes = [(L.OP_INPUT, -1, -1, 0, 1, 1, 1, 1, 0, 0, 0, 0),
                     (L.OP_CONV, 0, -1, c_out, 1, 1, 1, 1, 0, 0, affine, 0)]
            return L.lrcnn_plan(nodes, 1, c_in, rows, 1, dtype, L.CARRY, 1)
        self.fwd, self.bwd = plan(n_in, n_out, 1), plan(n_out, n_in, 0)
        need = max(self.fwd.info()["workspace_bytes"], self.bwd.info()["workspace_bytes"],
                   L.lrcnn_linear_wgrad_workspace_bytes(rows, n_in, n_out, dtype), 256)
        self.ws = torch.empty(need, device=device, dtype=torch.uint8)

    def forward(self, x, y):
        L.lrcnn_forward_rows(self.fwd, x, [None, self.w], [None, self.one], [None, self.b], y,
                             self.ws)

    def input_gradient(self, dy, dx):
        L.lrcnn_forward_rows(self.bwd, dy, [None, self.wt], [None, None], [None, None], dx,
                             self.ws)

    def weight_gradient(self, dy, ckpt, scale=None, shift=None):
        """dW and db from the checkpoint of the input (scale * it + shift)."""
        L.lrcnn_linear_wgrad(dy, ckpt, self.dw, self.ws, db=self.db, scale=scale, shift=shift)

    def update(self, lr):
        L.lrcnn_sgd_update(self.fwd, lr, [None, self.w], [None, self.dw])
        self.wt.copy_(self.w.t())
        self.b.sub_(lr * self.db)


class Norm:
    """Layer norm whose backward pass reads the checkpoint of its normalised rows."""

    def __init__(self, rows, cols, device):
        self.gamma = torch.ones(cols, device=device)
        self.beta = torch.zeros(cols, device=device)
        self.dgamma, self.dbeta = torch.empty(2, cols, device=device).unbind(0)
        self.rstd = torch.empty(rows, device=device)
        self.ckpt = torch.empty(L.lrcnn_act8_bytes(rows, cols), device=device, dtype=torch.uint8)
        self.ws = torch.empty(L.lrcnn_layer_norm_workspace_bytes(rows, cols), device=device,
                              dtype=torch.uint8)

    def forward(self, x, y, residual=None):
        L.lrcnn_layer_norm_forward(x, self.gamma, self.beta, EPS, y, residual=residual,
                                   rstd=self.rstd, ckpt=self.ckpt)

    def backward(self, dy, dx, dres=None):
        L.lrcnn_layer_norm_backward(dy, self.rstd, self.gamma, dx, self.dgamma, self.dbeta,
                                    self.ws, ckpt=self.ckpt, dres=dres)

    def update(self, lr):
        self.gamma.sub_(lr * self.dgamma)
        self.beta.sub_(lr * self.dbeta)


class GroupNorm:
    """Group norm with an activation over a map [batch * pixels][cols], whose backward
    pass reads the checkpoint of the normalised map."""

    def __init__(self, batch, pixels, cols, groups, kind, device="cuda"):
        self.batch, self.groups, self.kind = batch, groups, kind
        self.gamma = torch.ones(cols, device=device)
        self.beta = torch.zeros(cols, device=device)
        self.dgamma, self.dbeta = torch.empty(2, cols, device=device).unbind(0)
        self.rstd = torch.empty(batch, groups, device=device)
        self.ckpt = torch.empty(L.lrcnn_act8_bytes(batch * pixels, cols), device=device,
                                dtype=torch.uint8)
        self.ws = torch.empty(L.lrcnn_group_norm_workspace_bytes(batch, pixels, cols, groups),
                              device=device, dtype=torch.uint8)

    def forward(self, x, y):
        L.lrcnn_group_norm_forward(self.kind, x, self.gamma, self.beta, EPS, y, self.batch,
                                   self.groups, self.ws, rstd=self.rstd, ckpt=self.ckpt)

    def backward(self, dy, dx):
        L.lrcnn_group_norm_backward(self.kind, dy, self.rstd, self.gamma, self.beta, dx,
                                    self.batch, self.groups, self.ws, dgamma=self.dgamma,
                                    dbeta=self.dbeta, ckpt=self.ckpt)

    def update(self, lr):
        self.gamma.sub_(lr * self.dgamma)
        self.beta.sub_(lr * self.dbeta)


class Scratch:
    """Named byte buffers that blocks use within a pass and keep nothing in: one set
    for all blocks that run one after the other on one stream."""

    def __init__(self, sizes, device):
        self.buffers = {k: torch.empty(n, device=device, dtype=torch.uint8)
                        for k, n in sizes.items()}

    def take(self, name, *shape, dtype=torch.uint8):
        """The head of a buffer as a tensor."""
        n = math.prod(shape) * dtype.itemsize
        have = self.buffers[name].numel() if name in self.buffers else 0
        if n > have:
            raise ValueError(f"scratch for {name} has {have} bytes, {n} needed: make the largest "
                             "block first, one with dropout before one without")
        return self.buffers[name][:n].view(dtype).view(shape)


class FeedForward:
    """The block on [rows][cols] with `hidden` features in the middle. `scratch`: that
    of another block, at least as large, that runs before or after this one
    on the same stream; None: its own. `fused` (a gated block): two kernels a pass.
    `dropout`: the share of z that is dropped; `rng` (int64 [2] on the device): seed and
    offset of its generator, the offset advanced by the caller between steps, not between
    a step's forward and backward pass; `site`: another number for each block of a
    step."""

    def __init__(self, rows, cols, hidden, dtype=L.BF16, kind=L.ACT_GELU, gated=False,
                 device="cuda", seed=0, scratch=None, fused=False, dropout=0.0, rng=None, site=0):
        if fused and not gated:
            raise ValueError("a fused block is gated")
        if dropout and rng is None:
            raise ValueError("dropout needs rng")
        g = torch.Generator().manual_seed(seed)
        self.fused, self.dropout, self.rng, self.site = fused, dropout, rng, site
        self.kind, self.gated, self.hidden = kind, gated, hidden
        wide = 2 * hidden if gated else hidden
        self.norm1, self.norm2 = Norm(rows, cols, device), Norm(rows, cols, device)
        self.lin1 = Linear(rows, cols, wide, dtype, device, g)
        self.lin2 = Linear(rows, hidden, cols, dtype, device, g)

        def ckpt():
            return torch.empty(L.lrcnn_act8_bytes(rows, hidden), device=device, dtype=torch.uint8)
        # kept from forward to backward: the norms' and these checkpoints
        self.k_u, self.k_v = ckpt(), ckpt() if gated else None
        # scratch of both passes
        layers = (self.norm1, self.norm2, self.lin1, self.lin2)
        tdt, n_ws = torch_dtype(dtype), max(layer.ws.numel() for layer in layers)
        full = {"h": cols, "z": cols, "u": wide, "a": hidden}
        if dropout:
            full["d"] = cols  # the gradient behind the dropout
        if scratch is None:
            sizes = {k: rows * w * tdt.itemsize for k, w in full.items()}
            sizes.update(k_a=L.lrcnn_act8_bytes(rows, hidden), ws=n_ws)
            scratch = Scratch(sizes, device)
        self.scratch = scratch
        self.h, self.z, self.u, self.a, *self.d = (scratch.take(k, rows, w, dtype=tdt)
                                                   for k, w in full.items())
        self.k_a = scratch.take("k_a", L.lrcnn_act8_bytes(rows, hidden))
        scratch.take("ws", n_ws)
        for layer in layers:
            layer.ws = scratch.buffers["ws"]

    def saved_bytes(self):
        """Bytes kept from the forward to the backward pass."""
        kept = [self.norm1.ckpt, self.norm2.ckpt, self.norm1.rstd, self.norm2.rstd, self.k_u,
                self.k_v]
        return sum(t.numel() * t.element_size() for t in kept if t is not None)

    def _halves(self, t):
        return (t[:, :self.hidden], t[:, self.hidden:]) if self.gated else (t, None)

    def forward(self, x, y):
        u, v = self._halves(self.u)
        self.norm1.forward(x, self.h)
        if self.fused:
            L.lrcnn_gated_ffn_forward(self.kind, self.h, self.lin1.w, self.a, b1=self.lin1.b,
                                      w2=self.lin2.w, b2=self.lin2.b, z=self.z, ckpt_u=self.k_u,
                                      ckpt_v=self.k_v)
        else:
            self.lin1.forward(self.h, self.u)
            L.lrcnn_activation_forward(self.kind, u, self.a, v=v, ckpt_u=self.k_u,
                                       ckpt_v=self.k_v)
            self.lin2.forward(self.a, self.z)
        if self.dropout:
            L.lrcnn_dropout(self.z, self.z, self.dropout, self.rng, residual=x, site=self.site)
            self.norm2.forward(self.z, y)
        else:
            self.norm2.forward(self.z, y, residual=x)

    def backward(self, dy, dx):
        """dx from dy; the parameters' gradients stay with their layers."""
        du, dv = self._halves(self.u)
        dt, da, dh = self.z, self.a, self.h
        self.norm2.backward(dy, dt)
        dz = dt
        if self.dropout:
            dz = self.d[0]
            L.lrcnn_dropout(dt, dz, self.dropout, self.rng, site=self.site)
        if self.fused:
            L.lrcnn_gated_ffn_backward(self.kind, dz, self.lin2.wt, self.u, ckpt_u=self.k_u,
                                       ckpt_v=self.k_v, ckpt_a=self.k_a, w1t=self.lin1.wt, dx=dh)
            self.lin2.weight_gradient(dz, self.k_a)
        else:
            self.lin2.input_gradient(dz, da)
            L.lrcnn_activation_backward(self.kind, da, du, ckpt_u=self.k_u, ckpt_v=self.k_v,
                                        dv=dv, ckpt_a=self.k_a)
            self.lin2.weight_gradient(dz, self.k_a)
            self.lin1.input_gradient(self.u, dh)
        self.lin1.weight_gradient(self.u, self.norm1.ckpt, self.norm1.gamma, self.norm1.beta)
        self.norm1.backward(dh, dx, dres=dt)

    def update(self, lr):
        for layer in (self.norm1, self.norm2, self.lin1, self.lin2):
            layer.update(lr)


def main(fused=False):
    from .device import DeviceModel
    from .train import Trainer
    import numpy as np
    rng = np.random.default_rng(0)
    batch, size, classes, lr, steps = 16, 32, 10, 1e-3, 40
    conv = lambda src, c: (L.OP_CONV, src, -1, c, 3, 3, 1, 1, 1, 1, 0, 1)
    pool = lambda src: (L.OP_MAXPOOL, src, -1, 0, 2, 2, 2, 2, 0, 0, 0, 0)
    nodes = [(L.OP_INPUT, -1, -1, 0, 1, 1, 1, 1, 0, 0, 0, 0), conv(0, 32), pool(1), conv(2, 64),
             pool(3)]
    plan = L.lrcnn_plan(nodes, batch, 3, size, size, L.BF16, L.CARRY, 4)
    ws = [rng.standard_normal((32, 3, 3, 3)) * 0.2, None, rng.standard_normal((64, 3, 3, 32)) * 0.06,
          None]
    none = [None] * 4
    dm = DeviceModel(nodes, rng.standard_normal((batch, size, size, 3)), ws, none, none, L.BF16)
    oh, ow, oc = plan.node_shape(plan.n - 1)
    rows = batch * oh * ow
    fc = rng.standard_normal((classes, oh * ow * oc)) / math.sqrt(oh * ow * oc)
    tr = Trainer(plan, dm, fc, np.zeros(classes), rng.integers(0, classes, batch))
    more = {}
    if fused:
        state = torch.tensor([1, 0], device="cuda")
        more = dict(fused=True, dropout=0.1, rng=state)
        norm = GroupNorm(batch, oh * ow, oc, 8, L.ACT_SILU)
        n, dn = (torch.empty(rows, oc, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    block = FeedForward(rows, oc, 4 * oc, L.BF16, L.ACT_SILU, gated=True, **more)
    y, dy, dx = (torch.empty(rows, oc, device="cuda", dtype=torch.bfloat16) for _ in range(3))
    full = 2 * rows * (3 * oc + 3 * 4 * oc)
    print(f"{rows} rows of {oc}: {block.saved_bytes()} bytes kept, {full} in bfloat16")
    for step in range(steps):
        L.lrcnn_forward_rows(plan, dm.x, dm.w, dm.sc, dm.sf, tr.y, tr.ws)
        x = tr.y.view(rows, oc)
        if fused:
            state[1] = step
            norm.forward(x, n)
            block.forward(n, y)
        else:
            block.forward(x, y)
        L.lrcnn_head_loss(plan, y, tr.fc_w, tr.fc_b, tr.labels, tr.logits, tr.loss, dy,
                          tr.d_fc_w, tr.d_fc_b, tr.head_ws)
        if fused:
            block.backward(dy, dn)
            norm.backward(dn, dx)
            norm.update(lr)
        else:
            block.backward(dy, dx)
        L.lrcnn_backward_rows(plan, dm.x, dm.w, dm.sc, dm.sf, dx, dm.dw, None, tr.ws)
        L.lrcnn_sgd_update(plan, lr, dm.w, dm.dw, tr.fc_w, tr.d_fc_w, tr.fc_b, tr.d_fc_b)
        block.update(lr)
        if step % 5 == 0 or step == steps - 1:
            print(f"step {step}: loss {tr.loss[0].item():.4f}")


if __name__ == "__main__":
    import sys
    main(fused="--fused" in sys.argv[1:])
