"""The feed-forward example: a training step and served tokens against the same block in FP32."""
import pytest

from tests.gpu_util import dev, torch
from tests.libqe import need_lib

pytestmark = pytest.mark.gpu


def off(got, want):
    return float((got.float() - want).norm() / want.norm())


@pytest.mark.parametrize("tokens,hidden,ffn", [(256, 256, 512), (200, 192, 333)])
def test_step_is_near_fp32(tokens, hidden, ffn):
    """FP8 operands carry 3 (E4M3) or 2 (E5M2) mantissa bits: relative rounding errors uniform in +-2^-4 (+-2^-3) of a
    binade, rms 2^-4 / sqrt(3) = 0.036 and 0.072 at most.  A product of two rounded operands is off by the root of
    their squares' sum: 0.051 (E4M3 twice), 0.081 (E5M2 by E4M3).  y: h from G and U (0.051 each, through slopes of
    order 1: 0.1), rounded (0.036), times rounded Wd (0.036), beside the exact residual.  dx and dW: dy, Wd, dg / du
    (E5M2 again), the 8-bit G and U (0.3 steps of 1/63: below 0.01) and W or x: the root of the squares of 0.081,
    0.1, 0.072 and 0.036 is 0.15.  Bounds: 0.15 for y, 0.2 for the gradients."""
    need_lib()
    dev()
    from examples import gated_ffn
    block, x, dy = gated_ffn.make(tokens, hidden, ffn)
    y = block.forward(x).clone()
    dx, dwgu, dwd = block.backward(dy)
    want = gated_ffn.reference(block, x, dy)
    assert off(y, want[0]) < 0.15
    for got, ref in zip((dx, dwgu, dwd), want[1:]):
        assert off(got, ref) < 0.2
    # the residual is carried in its own precision: what is left of y is the block's output
    assert off(y.float() - x.float(), want[0] - x.float()) < 0.15
    # tokens served one by one (no scale moves) give the same codes, so the same sums up to FP32 order and one rounding
    a = block.serve(x[:1]).clone()
    b = block.serve(x[:16]).clone()
    assert off(b[:1], a.float()) < 0.01
    assert off(b, want[0][:16]) < 0.15


def test_steps_repeat_bit_for_bit():
    need_lib()
    dev()
    from examples import gated_ffn
    runs = []
    for _ in range(2):
        block, x, dy = gated_ffn.make(130, 160, 200, seed=3)
        runs.append([t.clone() for t in (block.forward(x), *block.backward(dy), block.codes, block.exps)])
    assert all(torch.equal(a, b) for a, b in zip(*runs))
