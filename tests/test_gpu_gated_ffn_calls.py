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
