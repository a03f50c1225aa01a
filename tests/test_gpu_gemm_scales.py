"""FP8 products whose scale inverses are not powers of two, on the GPU.

Operands are codes of small integers, so every sum is an exact integer below 2^24; with u = 2^-24 the product of the
two inverses and its product with the sum are off by u each, a gated output by the same for either projection and u
for their product, and a BF16 output by another half ulp (2^-8 of the value at most)."""
import math

import numpy as np
import pytest

from oracle import fp8
from tests.gpu_util import dev, torch
from tests.libqe import need_lib

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SHAPES = [(1, 40, 100), (16, 64, 2100), (65, 62, 600), (129, 200, 130), (300, 520, 384)]
SCALES = [(0.75, 1.0), (1.0 / 3.0, 3.7 / 448.0), (-0.625, 1.9), (-1.0, 0.5), (1.1 * 2.0 ** -120, 1.7 * 2.0 ** 119),
          (1.3 * 2.0 ** 126, 1.5 * 2.0 ** -126), (0.0, 3.0), (0.25, 8.0)]


def codes(rng, rows, k, d):
    v = rng.integers(-6, 7, size=(rows, k))
    q = np.zeros((rows, (k + 15) // 16 * 16), dtype=np.uint8)
    q[:, :k] = fp8.encode(v.astype(np.float64), "E4M3")
    return torch.from_numpy(q).to(d), v.astype(np.float64)


def near(got, want, rounds, bf16=False):
    off = np.abs(got.double().cpu().numpy() - want)
    assert (off <= np.abs(want) * (rounds * U * 1.01 + (2.0 ** -8 if bf16 else 0.0))).all(), off.max()


def each_tile(qe, names):
    for name in names:
        assert qe.qe_set_gemm_tile(getattr(qe, name)) == "OK"
        try:
            yield name
            torch.cuda.synchronize()
        finally:
            assert qe.qe_set_gemm_tile(qe.TILE_AUTO) == "OK"


@pytest.mark.parametrize("scales", SCALES, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_plain_product(shape, scales):
    qe, d = need_lib(), dev()
    m, n, k = shape
    rng = np.random.default_rng(m)
    (a, av), (b, bv) = codes(rng, m, k, d), codes(rng, n, k, d)
    s = torch.tensor(scales, dtype=torch.float32, device=d)
    sa, sb = (float(v) for v in s)
    want = av @ bv.T * (sa * sb)
    for _ in each_tile(qe, ["TILE_AUTO", "TILE_256x256", "TILE_256x224", "TILE_256x192", "TILE_192x256", "TILE_256x128"]):
        for dt, q in ((torch.float32, qe.F32), (torch.bfloat16, qe.BF16)):
            c = torch.zeros((m, n), dtype=dt, device=d)
            assert qe.qe_fp8_gemm_tn(a, 0, a.shape[1], b, 0, b.shape[1], m, n, k, s[0:1], s[1:2], c, q, n, qe.INIT) == "OK"
            near(c, want, 2, q == qe.BF16)
        c = torch.zeros((m, n), device=d)
        for mode in (qe.INIT, qe.ACCUM):
            assert qe.qe_fp8_gemm_tn(a, 0, a.shape[1], b, 0, b.shape[1], m, n, k, s[0:1], s[1:2], c, qe.F32, n, mode) == "OK"
        near(c, 2 * want, 3)


@pytest.mark.parametrize("scales", SCALES, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_product_with_an_epilogue(shape, scales):
    """Bias and activation see the scaled sum: relu(Z + 0) and the value saved for the backward pass."""
    qe, d = need_lib(), dev()
    m, n, k = shape
    rng = np.random.default_rng(n)
    (a, av), (b, bv) = codes(rng, m, k, d), codes(rng, n, k, d)
    s = torch.tensor(scales, dtype=torch.float32, device=d)
    z = av @ bv.T * (float(s[0]) * float(s[1]))
    for _ in each_tile(qe, ["TILE_AUTO", "TILE_256x256", "TILE_192x256"]):
        c, keep = torch.zeros((m, n), device=d), torch.zeros((m, n), dtype=torch.bfloat16, device=d)
        bias = torch.zeros(n, device=d)
        epi = qe.make_epilogue(qe.ACT_RELU, bias, qe.F32, saved=qe.make_saved(qe.SAVED_BF16, keep, n))
        assert qe.qe_fp8_gemm_act(a, 0, a.shape[1], b, 0, b.shape[1], m, n, k, s[0:1], s[1:2], epi, c, qe.F32, n) == "OK"
        near(c, np.maximum(z, 0.0), 2)
        near(keep, z, 2, True)


@pytest.mark.parametrize("scales", SCALES, ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_gated_product(shape, scales):
    """The two projections have factors of their own."""
    qe, d = need_lib(), dev()
    m, n, k = shape
    rng = np.random.default_rng(k)
    (a, av), (w, wv) = codes(rng, m, k, d), codes(rng, 2 * n, k, d)
    s = torch.tensor([0.7, *scales], dtype=torch.float32, device=d)
    if abs(math.log2(abs(scales[0]) + 1e-30)) > 40:
        s[1], s[2] = s[1] * 2.0 ** (-100 if scales[0] > 1 else 100), s[2] * 2.0 ** (100 if scales[0] > 1 else -100)
    sx, sg, su = (float(v) for v in s)
    want = (av @ wv[:n].T * (sx * sg)) * (av @ wv[n:].T * (sx * su))
    for _ in each_tile(qe, ["TILE_AUTO", "TILE_256x256", "TILE_192x256"]):
        h = torch.zeros((m, n), device=d)
        assert qe.qe_fp8_gemm_gated(a, 0, a.shape[1], w, w[n:], 0, w.shape[1], m, n, k, s[0:1], s[1:2], s[2:3], qe.ACT_NONE, h,
                                    qe.F32, n) == "OK"
        near(h, want, 5)


def test_a_nan_scale_is_not_lost():
    qe, d = need_lib(), dev()
    rng = np.random.default_rng(1)
    (a, _), (b, _) = codes(rng, 20, 64, d), codes(rng, 40, 64, d)
    s = torch.tensor([math.nan, 1.0], device=d)
    c = torch.zeros((20, 40), device=d)
    assert qe.qe_fp8_gemm_tn(a, 0, 64, b, 0, 64, 20, 40, 64, s[0:1], s[1:2], c, qe.F32, 40, qe.INIT) == "OK"
    assert bool(c.isnan().all())
    assert qe.qe_fp8_gemm_act(a, 0, 64, b, 0, 64, 20, 40, 64, s[1:2], s[0:1], None, c.zero_(), qe.F32, 40) == "OK"
    assert bool(c.isnan().all())


@pytest.mark.parametrize("exps", [(-126, -19), (-100, -45), (-140, 100), (-126, -126), (100, 20), (126, -126), (64, -64), (-3, 7)], ids=str)
def test_powers_of_two_round_once(exps):
    """Results that are denormal, zero or infinite too are what one rounding of the exact product gives."""
    qe, d = need_lib(), dev()
    m, n, k = 70, 80, 200
    rng = np.random.default_rng(2)
    (a, av), (b, bv) = codes(rng, m, k, d), codes(rng, n, k, d)
    s = torch.tensor([2.0 ** e for e in exps], dtype=torch.float32, device=d)
    with np.errstate(over="ignore"):
        want = (av @ bv.T * 2.0 ** sum(exps)).astype(np.float32)
    for _ in each_tile(qe, ["TILE_AUTO", "TILE_256x256"]):
        c = torch.zeros((m, n), device=d)
        assert qe.qe_fp8_gemm_tn(a, 0, a.shape[1], b, 0, b.shape[1], m, n, k, s[0:1], s[1:2], c, qe.F32, n, qe.INIT) == "OK"
        assert np.array_equal(c.cpu().numpy(), want)
        assert qe.qe_fp8_gemm_act(a, 0, a.shape[1], b, 0, b.shape[1], m, n, k, s[0:1], s[1:2], None, c.zero_(), qe.F32, n) == "OK"
        assert np.array_equal(c.cpu().numpy(), want)
    c = torch.zeros((5, n), device=d)
    assert qe.qe_fp8_gemm_act(a, 0, a.shape[1], b, 0, b.shape[1], 5, n, k, s[0:1], s[1:2], None, c, qe.F32, n) == "OK"
    assert np.array_equal(c.cpu().numpy(), want[:5])
