"""Which kernels the operators between the linears take on devices with other numbers of compute units (fake HIP runtime)."""
import pytest

from tests.fake_hip import ADDR, calls


def product(qe, hip, cases):
    got = []
    for gated, m, n, k in cases:
        hip.clear()
        ld = (k + 15) // 16 * 16
        if gated:
            st = qe.qe_fp8_gemm_gated(ADDR, 0, ld, ADDR, ADDR, 0, ld, m, n, k, ADDR, ADDR, ADDR, qe.ACT_SILU, ADDR, qe.BF16,
                                      n, stream=0)
        else:
            st = qe.qe_fp8_gemm_act(ADDR, 0, ld, ADDR, 0, ld, m, n, k, ADDR, ADDR, None, ADDR, qe.BF16, n, stream=0)
        assert st == "OK", st
        got.append("act_rows_kernel" in hip.log("launch")[0][2])
    return got


def gradient(qe, hip, cases):
    got = []
    for rows, cols in cases:
        hip.clear()
        z = qe.make_saved(qe.SAVED_I8, ADDR, cols, ADDR, (cols + 31) // 32)
        st = qe.qe_act_grad(ADDR, qe.BF16, cols, rows, cols, qe.ACT_SILU, z, dz=ADDR, ld_dz=cols, stream=0)
        assert st == "OK", st
        got.append("ELi64ELi512E" in hip.log("launch")[0][2])
    return got


@pytest.mark.parametrize("units", [64, 256])
def test_limits_follow_the_compute_units(units, monkeypatch):
    """One 16 x 16 block a unit (two from K = 12289 on, not for gated products); four 128 x 128 tiles a unit."""
    monkeypatch.setenv("FAKE_HIP_UNITS", str(units))
    n = units  # 16 columns of blocks for 256 units, 4 for 64: 16 row blocks fill the units
    assert calls(product, [[False, 256, n, 1025], [False, 257, n, 1025], [True, 256, n, 1025], [True, 257, n, 1025],
                           [False, 512, n, 12289], [False, 513, n, 12289], [True, 512, n, 12289]]) == [True, False, True, False,
                                                                                                        True, False, False]
    assert calls(product, [[False, 16, 64 * units, 1025], [True, 1, 4096, 128]]) == [True, True]  # up to 16 rows: always
    assert calls(gradient, [[512, 128 * units], [513, 128 * units]]) == [True, False]


def saves(qe, hip, cases):
    got = []
    for rows, cols, dtype in cases:
        hip.clear()
        s = qe.make_saved(qe.SAVED_I8, ADDR, cols, ADDR, (cols + 31) // 32)
        assert qe.qe_act_save(ADDR, dtype, cols, rows, cols, s, stream=0) == "OK"
        got.append(hip.log("launch")[0][2])
    return got


def test_saves_of_every_size_take_one_kernel_a_type():
    """A saved tensor is read again: no size has loads that keep it out of the caches."""
    for dtype in (0, 1):
        assert len(set(calls(saves, [[1, 32, dtype], [1500, 4099, dtype], [4096, 14336, dtype], [8192, 28672, dtype]]))) == 1
