"""The float64 definitions of block-scaled codes and of the norms around a residual sum."""
import numpy as np
import pytest

from oracle import blocks as ob
from oracle import fp8


@pytest.mark.parametrize("fmt,fmax,half", [("E4M3", 448.0, 2.0 ** -4), ("E5M2", 57344.0, 2.0 ** -3)])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_blocks_restore_within_half_a_step(fmt, fmax, half, block_rows):
    rng = np.random.default_rng(1)
    x = rng.normal(size=(130, 300)) * np.exp(rng.normal(size=(130, 1)))
    codes, exps = ob.pack(x, fmt, block_rows)
    assert exps.shape == (-(-130 // block_rows), 3)
    back = ob.unpack(codes, exps, fmt, block_rows)
    low = {"E4M3": 2.0 ** -10, "E5M2": 2.0 ** -17}[fmt]  # half the smallest step of the format
    for i in range(exps.shape[0]):
        for b in range(3):
            at = np.s_[i * block_rows:(i + 1) * block_rows, b * 128:(b + 1) * 128]
            step = 2.0 ** (int(exps[i, b]) - 127)
            a = np.abs(x[at]).max() / step
            assert fmax / 2 < a <= fmax  # the largest power of two that does not saturate
            assert (np.abs(back[at] - x[at]) <= np.maximum(half * np.abs(x[at]), low * step)).all()


@pytest.mark.parametrize("amax,fmt,byte", [(448.0, "E4M3", 127), (448.0000305, "E4M3", 128), (1.0, "E4M3", 119), (0.0, "E4M3", 1),
                                           (2.0 ** -140, "E4M3", 1), (3.4028235e38, "E4M3", 247), (57344.0, "E5M2", 127),
                                           (57345.0, "E5M2", 128), (1.75, "E5M2", 112), (np.inf, "E4M3", 255), (np.nan, "E5M2", 255)])
def test_exponent_byte(amax, fmt, byte):
    x = np.zeros((2, 130), dtype=np.float32)
    x[1, 129] = -amax
    codes, exps = ob.pack(x, fmt)
    assert exps.tolist() == [[1, 1], [1, byte]]
    assert np.isnan(fp8.decode(codes[1, 128:], fmt)).all() == (byte == 255)
    assert ob.pack(x, fmt, 128)[1].tolist() == [[1, byte]]


CASES = [dict(), dict(x_scale=0.5, y_scale=0.25, post=True), dict(post=True, gate_rows=2, gate=True), dict(gate=True, gate_rows=3),
         dict(no_x=True, post=True), dict(no_y=True, x_scale=2.0), dict(no_dr=True, post=True), dict(no_dh=True, post=True, gate=True)]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_gradient_is_the_difference_quotient(case):
    """Of f = sum dr r + sum dh h, against central differences with step 1e-5: truncation h^2 f''' and rounding eps f / h are below 1e-9."""
    rng = np.random.default_rng(5)
    rows, cols = 5, 7
    v = {k: rng.normal(size=(rows, cols)) for k in ("x", "y", "dr", "dh")}
    v.update(post=1 + 0.1 * rng.normal(size=cols), pre=1 + 0.1 * rng.normal(size=cols))
    gate_rows = case.get("gate_rows", rows)
    v["gate"] = rng.normal(size=(-(-rows // gate_rows), cols))
    have = {k: not case.get("no_" + k, False) for k in ("x", "y", "dr", "dh")}
    have.update(post=case.get("post", False), gate=case.get("gate", False), pre=have["dh"])
    eps = 0.01
    opt = dict(x_scale=case.get("x_scale", 1.0), y_scale=case.get("y_scale", 1.0), gate_rows=gate_rows)

    def args(v):
        return dict(post=v["post"] if have["post"] else None, post_eps=eps if have["post"] else None,
                    gate=v["gate"] if have["gate"] else None, **opt)

    def r_of(v):
        return ob.residual(v["x"] if have["x"] else None, v["y"] if have["y"] else None, **args(v))

    def f(v):
        r = r_of(v)
        return (v["dr"] * r).sum() * have["dr"] + (v["dh"] * ob.norm(r, eps, v["pre"])).sum() * have["dh"]
    got = ob.residual_grad(v["dr"] if have["dr"] else None, v["dh"] if have["dh"] else None, r_of(v), v["y"] if have["y"] else None,
                           pre=v["pre"], pre_eps=eps, **args(v))
    names = {"x": "dx", "y": "dy", "post": "dpost", "pre": "dpre", "gate": "dgate"}
    for name, g in names.items():
        if not have[name]:
            continue
        want = np.zeros_like(v[name])
        for i in np.ndindex(want.shape):
            a, b = dict(v, **{name: v[name].copy()}), dict(v, **{name: v[name].copy()})
            a[name][i] += 1e-5
            b[name][i] -= 1e-5
            want[i] = (f(a) - f(b)) / 2e-5
        assert np.abs(got[g] - want).max() < 1e-7, name
