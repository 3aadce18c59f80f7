"""The parameters' gradients of the group norm over very many images, whose terms cancel.

Tolerance. With one pixel an image, no activation and a checkpoint, what an image adds is
exact in float32: dy for dbeta; for dgamma dy times a checkpoint's value, 8 bits times 7.
N images' terms are added in 64 bits, at most N / 32 one after another and 32 joins: off by
at most (N / 32 + 32) 2^-53 of the sum of their magnitudes, and rounded once, 2^-24 of the
result. (Added in float32 they were off by up to 290 times this.) Added to what is there: one
more term, the same rounding."""
import math

import pytest
import torch

from paper_2401_11471_amd import lrcnn as L

pytestmark = pytest.mark.gpu


def cancelling(n, cols, g):
    """Values of very different size, each of the first half with its negative in the second,
    in another order; the last one of every column has none."""
    half = torch.randn(n // 2, cols, generator=g, device="cuda")
    half.mul_(torch.exp(2 * torch.randn(n // 2, cols, generator=g, device="cuda")))
    order = torch.randperm(n // 2, generator=g, device="cuda")
    both = torch.cat([half, -half[order]]).bfloat16()
    both[-1] += 0.5
    return both


@pytest.mark.parametrize("batch,cols,groups", [(1 << 18, 8, 2), ((1 << 16) + 3, 40, 5), (1000, 8, 8)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_gradients_of_many_images(batch, cols, groups, dtype):
    print("gradients of many images", batch, cols, groups, dtype, flush=True)
    g = torch.Generator(device="cuda").manual_seed(batch)
    dy = cancelling(batch, cols, g) if batch % 2 == 0 else \
        torch.cat([cancelling(batch - 1, cols, g), torch.ones(1, cols, device="cuda").bfloat16()])
    ck = torch.empty(L.lrcnn_act8_bytes(batch, cols), device="cuda", dtype=torch.uint8)
    L.lrcnn_act8_pack(torch.randn(batch, cols, generator=g, device="cuda"), ck)
    xh = torch.empty(batch, cols, device="cuda")
    L.lrcnn_act8_unpack(ck, xh)
    ws = torch.empty(L.lrcnn_group_norm_workspace_bytes(batch, 1, cols, groups), device="cuda",
                     dtype=torch.uint8)
    dy, dx = dy.to(dtype), torch.empty(batch, cols, device="cuda", dtype=dtype)
    rstd = torch.ones(batch, groups, device="cuda")
    terms = {"dgamma": dy.double() * xh.double(), "dbeta": dy.double()}
    for old in (None, 0.375):
        out = {k: torch.full((cols,), math.nan if old is None else old, device="cuda") for k in terms}
        L.lrcnn_group_norm_backward(L.ACT_NONE, dy, rstd, None, None, dx, batch, groups, ws, ckpt=ck,
                                    accumulate=old is not None, **out)
        for k, t in terms.items():
            t = t.cpu()
            ref = torch.tensor([math.fsum(c.tolist() + [old or 0.0]) for c in t.t()],
                               dtype=torch.float64)
            tol = 2.0 ** -24 * ref.abs() + (batch / 32 + 33) * 2.0 ** -53 * t.abs().sum(0)
            off = (out[k].double().cpu() - ref).abs()
            assert (off <= tol).all(), (k, old, float((off / tol).max()))
