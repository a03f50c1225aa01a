"""What the feed-forward example refuses, and that serving leaves training alone."""
import pytest

from tests.gpu_util import dev, torch
from tests.libqe import need_lib

pytestmark = pytest.mark.gpu


def made(tokens=130, hidden=160, ffn=200, seed=3):
    need_lib()
    dev()
    from examples import gated_ffn
    return gated_ffn.make(tokens, hidden, ffn, seed)


def test_tensors_of_other_sizes_and_types_are_refused():
    """Nothing is enqueued for them: they would be read, or the block's buffers written, past their ends."""
    from examples import gated_ffn
    block, x, dy = made()
    more = torch.cat((x, x[:1]))
    for bad in (more, x[:129], x.float(), x[:, :159].contiguous(), x.t().contiguous().t(), x.cpu(), x[::2]):
        with pytest.raises(ValueError):
            block.forward(bad)
        with pytest.raises(ValueError):
            block.backward(bad)
    for bad in (more, x[:5].float(), x[:5, :159].contiguous(), x[:, ::2][:5], x[0]):
        with pytest.raises((ValueError, IndexError)):
            block.serve(bad)
    with pytest.raises(ValueError):
        gated_ffn.GatedFFN(block.wgu_master[:-1], block.wd_master, 8)
    with pytest.raises(ValueError):
        gated_ffn.GatedFFN(block.wgu_master.half(), block.wd_master, 8)
    assert block.serve(x).shape == x.shape and block.serve(x[:0]).shape == (0, 160)


def test_serving_leaves_training_alone():
    """Two steps with tokens served between each forward and its backward, and after them, equal the same steps without, bit
    for bit: gradients, histories, scales and what the next step makes of them.  The served tokens' amax is 64 times
    training's, and the second step's input 8 times the first's, so that its scales move."""
    runs = []
    for serving in (False, True):
        block, x, dy = made()
        kept = []
        for step in range(3):
            xs = x * (8 if step > 0 else 1)
            y = block.forward(xs).clone()
            if serving:
                block.serve((x * 64)[:17])
            kept += [y, *(t.clone() for t in block.backward(dy))]
            if serving:
                block.serve((x * 64)[:1])
            for role in (block.x, block.h_q, block.dy, block.dgu, block.wgu, block.wd):
                kept += [role.hist.clone(), role.scales.clone(), role.accum.clone(), role.row.clone(), role.col.clone()]
        runs.append(kept)
    assert len(runs[0]) == len(runs[1]) and all(torch.equal(a, b) for a, b in zip(*runs))
    assert not torch.equal(runs[0][5], runs[0][5 + 34])  # x's scale moved between the first and the second step


def test_served_tokens_are_the_trained_block_s():
    """At the same scales a served token is the forward's own row, up to the order of its sums and one rounding."""
    block, x, dy = made(tokens=64)
    y = block.forward(x).clone()
    block.backward(dy)
    got = block.serve(x).float()
    assert float((got - y.float()).norm() / y.float().norm()) < 0.01
