"""The gradient of the norms around a residual sum, on the host: how many workgroups its rows are given."""
import pytest

from tests.fake_hip import ADDR, calls


def grids(qe, hip, rows, cols, groups, sums):
    got = []
    for n in groups:
        hip.clear()
        ms = [qe.make_matrix(i * ADDR, cols, qe.BF16) for i in range(1, 7)]
        gate_rows = -(-rows // n)
        d = qe.make_residual(post_norm=True, post_weight=ADDR, pre_norm=True, pre_weight=ADDR, gate=ADDR, ld_gate=cols, gate_rows=gate_rows)
        out = [ADDR, 2 * ADDR, 3 * ADDR, qe.INIT, ADDR] if sums else [None, None, None, qe.INIT, None]
        assert qe.qe_residual_norm_grad(*ms[:4], rows, cols, d, ADDR, ADDR, *ms[4:], *out, stream=0) == "OK"
        got += [[-(-rows // gate_rows), int(w[3].split("=")[1])] for w in hip.log("launch") if "residual_grad_kernel" in w[2]]
    return got


@pytest.mark.parametrize("units", [64, 256])
@pytest.mark.parametrize("sums", [True, False], ids=["sums", "no_sums"])
def test_no_more_workgroups_than_units(units, sums, monkeypatch):
    """A unit holds one workgroup: with a few more than units, those left over would run when the others have ended, and the
    whole call would take twice as long.  Groups of gates that are fewer than the units share them."""
    monkeypatch.setenv("FAKE_HIP_UNITS", str(units))
    groups = [1, 2, 3, 5, 6, 7, 8, 13, 31, 63, 64, 100, 200, 255, 256, 300]
    for n, workgroups in calls(grids, 8192, 8192, groups, sums):
        if n <= units:
            assert units // 2 < workgroups <= units, n  # (7 groups of 1171 rows: 252; 200: 200)
        else:
            assert workgroups == n
