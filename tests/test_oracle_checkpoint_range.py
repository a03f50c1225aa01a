"""The float64 checkpoint format at the top of the float32 range."""
import numpy as np
import pytest

from oracle import activation as oa

STEP = 2.0 ** 122  # the largest step


@pytest.mark.parametrize("value,code,byte", [(127 * 2.0 ** 120, 127, 247), (127 * 2.0 ** 121, 127, 248), (63.6 * STEP, 63, 249),
                                             (float(np.finfo(np.float32).max), 63, 249), (-63.9 * STEP, -63, 249)])
def test_finite_values_restore_to_finite_float32(value, code, byte):
    x = np.zeros((1, 40), dtype=np.float32)
    x[0, 7], x[0, 9] = value, 0.25 * value
    codes, exps = oa.pack(x)
    back = oa.unpack(codes, exps)
    assert codes[0, 7] == code and exps[0, 0] == byte and np.isfinite(back.astype(np.float32)).all()
    step = 2.0 ** (byte - 127)
    assert abs(back[0, 7] - x[0, 7]) < step and abs(back[0, 9] - x[0, 9]) <= step / 2
