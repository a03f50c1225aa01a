"""Workgroups of the norm around a residual sum that take three rows and more, one after the other: the next row is on its way
while this one is stored, sums go through buffers that take turns, gates change from row to row.  Against float64, with the
tolerances of test_gpu_residual_norm.py."""
import pytest

from tests.gpu_util import dev, torch
from tests.libqe import need_lib
from tests.test_gpu_residual_norm import Case

pytestmark = pytest.mark.gpu


def rows_for(cols, turns=2):
    """More than `turns` rows for each of the workgroups that a device is given: 2048 lanes a unit, in powers of two for a row."""
    lanes = 64
    while lanes * 8 < cols and lanes < 1024:
        lanes *= 2
    return turns * torch.cuda.get_device_properties(0).multi_processor_count * (2048 // lanes) + 37


# row lengths: a wave a row, four waves, sixteen with eight values a lane and with sixteen
FORMS = [dict(gate_rows=200, xs=0.875, ys=0.5), dict(x="f32", y="f32", r="f32", weights="f32", gate_rows=3, pad=1), dict(x="f32", r="f32", offset=1.0),
         dict(post=False, h="bf16", pad=3)]


@pytest.mark.parametrize("form", FORMS, ids=lambda f: "-".join(f"{k}{v}" for k, v in f.items()))
@pytest.mark.parametrize("cols", [70, 1040, 4104, 8200])
def test_three_rows_a_workgroup(cols, form):
    c = Case(need_lib(), dev(), rows_for(cols), cols, cols, **form)
    c.check_forward(*c.forward(row=0))


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [70, 4104, 8200])
def test_three_rows_in_place(cols, t):
    """r over x, held against float64; and h over y beside it, with the bits of h elsewhere."""
    qe, d = need_lib(), dev()
    form = dict(x=t, y=t, r=t, weights=t, gate_rows=100)
    c = Case(qe, d, rows_for(cols), cols, 1, **form)
    c.check_forward(*c.forward(row=0, in_place=True))
    a, b = (Case(qe, d, rows_for(cols), cols, 2, h=t, **form) for _ in range(2))
    a.forward()
    assert qe.qe_residual_norm(b.handle(b.x), b.handle(b.y), b.rows, cols, b.desc, b.handle(b.x), b.handle(b.y)) == "OK"
    torch.cuda.synchronize()
    assert torch.equal(a.r, b.x) and torch.equal(a.h, b.y)
