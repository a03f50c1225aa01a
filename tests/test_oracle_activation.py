"""The float64 activations, gradients and the 8-bit checkpoint format."""
import numpy as np
import pytest

from oracle import activation as oa

Z = np.concatenate([np.linspace(-12, 12, 481), [-1e-6, 0.25, 1e-6]])


@pytest.mark.parametrize("act", oa.ACTS)
def test_slope_is_the_difference_quotient(act):
    z = Z[np.abs(Z) > 1e-3] if act == "relu" else Z
    h = 1e-5
    quotient = (oa.value(z + h, act) - oa.value(z - h, act)) / (2 * h)
    # truncation h^2 / 6 max |f'''| < 1e-10, rounding 2 eps |f| / h < 6e-10
    assert np.abs(oa.slope(z, act) - quotient).max() < 2e-9


@pytest.mark.parametrize("act", oa.ACTS)
def test_gate_gradient_is_the_difference_quotient(act):
    rng = np.random.default_rng(3)
    g, u, dd = rng.normal(size=(3, 5, 7))
    g[np.abs(g) < 1e-3] = 0.5
    got, h = oa.gate_grad(dd, g, u, act), 1e-5
    dg = dd * (oa.gate(g + h, u, act) - oa.gate(g - h, u, act)) / (2 * h)
    du = dd * (oa.gate(g, u + h, act) - oa.gate(g, u - h, act)) / (2 * h)
    assert np.abs(got - np.concatenate([dg, du], 1)).max() < 1e-8


def test_known_values():
    assert oa.value(np.array([1.0]), "gelu")[0] == pytest.approx(0.8413447460685429, abs=1e-15)   # Phi(1)
    assert oa.value(np.array([0.0, -3.0, 3.0]), "relu").tolist() == [0.0, 0.0, 3.0]
    assert oa.value(np.array([0.0]), "silu")[0] == 0.0 and oa.slope(np.array([0.0]), "silu")[0] == 0.5


@pytest.mark.parametrize("amax,byte", [(127.0, 127), (127.0000076, 128), (1.0, 121), (1.984375, 121), (2.0, 122), (0.0, 1),
                                       (2.0 ** -130, 1), (3.0e38, 248), (np.float32(3.4028235e38), 249)])
def test_exponent_byte(amax, byte):
    x = np.zeros((1, 32), dtype=np.float32)
    x[0, 5] = -amax
    codes, exps = oa.pack(x)
    assert exps.tolist() == [[byte]] and abs(int(codes[0, 5])) <= 127


def test_round_trip_is_within_half_a_step_and_idempotent():
    rng = np.random.default_rng(1)
    x = (rng.normal(size=(40, 100)) * 10.0 ** rng.integers(-6, 7, size=(40, 1))).astype(np.float32)
    codes, exps = oa.pack(x)
    back = oa.unpack(codes, exps)
    step = np.repeat(2.0 ** (exps.astype(int) - 127.0), 32, axis=1)[:, :100]
    amax = np.repeat(np.stack([np.abs(x[:, g:g + 32]).max(1) for g in range(0, 100, 32)], 1), 32, axis=1)[:, :100]
    assert (np.abs(back - x) <= step / 2).all()
    assert (step <= amax / 63.5).all() and (step >= amax / 127 * (1 - 1e-7)).all()
    # restored values have seven significant bits: exact in bf16, and packing them again changes nothing
    assert (back.astype(np.float32).view(np.uint32) & 0xFFFF == 0).all()
    assert (oa.unpack(*oa.pack(back)) == back).all()


def test_groups_that_are_not_finite_restore_as_nan():
    x = np.ones((3, 70), dtype=np.float32)
    x[0, 3], x[1, 69] = np.inf, np.nan
    codes, exps = oa.pack(x)
    back = oa.unpack(codes, exps)
    assert exps[0].tolist() == [255, 121, 121] and exps[1].tolist() == [121, 121, 255]
    assert np.isnan(back[0, :32]).all() and np.isnan(back[1, 64:]).all() and (back[2] == 1).all()
