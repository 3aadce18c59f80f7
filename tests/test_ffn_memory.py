"""What feed-forward blocks with 8-bit checkpoints own: memory that a pass alone uses
exists once, however many blocks share it. Host code only (buffers in host memory,
never touched)."""
import pytest
import torch

from paper_2401_11471_amd import ffn
from paper_2401_11471_amd import lrcnn as L


def storages(*objs):
    """Bytes of the distinct buffers that objects hold, parameters among them."""
    seen, out, todo = set(), {}, list(objs)
    while todo:
        o = todo.pop()
        if isinstance(o, torch.Tensor):
            out[o.untyped_storage().data_ptr()] = o.untyped_storage().nbytes()
        elif type(o).__module__ == ffn.__name__ and id(o) not in seen:
            seen.add(id(o))
            todo += vars(o).values()
    return sum(out.values())


@pytest.mark.parametrize("gated", [False, True])
def test_blocks_share_their_scratch(gated):
    rows, cols, hidden = 20000, 256, 1024
    make = lambda **k: ffn.FeedForward(rows, cols, hidden, gated=gated, device="cpu", **k)
    first = make()
    blocks = [first] + [make(scratch=first.scratch) for _ in range(3)]
    wide = 2 * hidden if gated else hidden
    # w, wt and dw of both layers, and small vectors
    weights = (wide + hidden) * cols * (2 + 2 + 4) + (1 << 16)
    one = storages(first)
    for b in blocks[1:]:
        assert storages(first, b) - one <= b.saved_bytes() + weights
    # a bfloat16 block keeps x, h, x + z, u and a
    assert storages(*blocks) < len(blocks) * (rows * 2 * (3 * cols + hidden + wide) + weights)
    assert storages(*blocks) == one + sum(storages(first, b) - one for b in blocks[1:])


def test_scratch_of_a_larger_block_serves_a_smaller_one_only():
    big = ffn.FeedForward(1000, 96, 300, L.F32, gated=True, device="cpu")
    small = ffn.FeedForward(900, 64, 200, L.BF16, device="cpu", scratch=big.scratch)
    assert small.u.shape == (900, 200) and small.u.dtype is torch.bfloat16
    assert small.u.data_ptr() == big.u.data_ptr() and small.lin1.ws is big.lin2.ws
    for kw in (dict(rows=1100), dict(cols=128), dict(hidden=400)):
        a = dict(dict(rows=1000, cols=96, hidden=300), **kw)
        with pytest.raises(ValueError):
            ffn.FeedForward(a["rows"], a["cols"], a["hidden"], L.F32, gated=True, device="cpu",
                            scratch=big.scratch)
