"""Products with an epilogue, the gated feed-forward, the gradient through the activation and 8-bit checkpoints on the
GPU, against float64.

Operands are codes of small integers, so every sum is an integer below 2^24 and exact, and with a bias that is a multiple
of 2^-7 the pre-activation is exact too: what is saved has to be right bit for bit, and only the activation, one
FP32 product or sum and the final rounding may be off.  With u = 2^-24:
  value: 16 u (1 + |z|) (silu and gelu_tanh: an exponent's error |t| u matters only where e^-t does not vanish,
         t e^-t < 1, then four roundings; gelu: erf is within 2 u, times |z|);
  slope: (16 + 4 |z|) u, each of its terms being at most 1 and its exponents' errors as above;
  BF16 outputs: half an ulp more, at most 2^-8 of the value (8-bit significand), and 2^-10 of that for the FP32 error's
  tip over a tie.
"""
import math

import numpy as np
import pytest

from oracle import activation as oa
from oracle import fp8
from tests.act_tiles import TILES
from tests.gpu_util import accum_buffer, accum_value, dev, meta_buffer, meta_of, torch
from tests.libqe import need_lib

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
FMTS = ("E4M3", "E5M2")
ACT = {a: i for i, a in enumerate(oa.ACTS)}
SHAPES = [(1, 1, 1), (1, 32, 16), (2, 33, 100), (3, 31, 129), (16, 64, 128), (17, 130, 257), (37, 53, 100), (64, 64, 512),
          (65, 200, 130), (128, 256, 256), (255, 511, 129), (300, 520, 384), (1, 300, 1500), (5, 96, 4100), (513, 257, 1000)]
ids = lambda s: "x".join(map(str, s)) if isinstance(s, tuple) else None  # noqa: E731


def rup16(v):
    return (v + 15) // 16 * 16


def int_codes(rng, rows, k, fmt, d):
    """Codes of integers in -6 .. 6 with other (finite) codes behind column k, and the integers, on the device."""
    v = rng.integers(-6, 7, size=(rows, k))
    q = np.full((rows, rup16(k)), 0x3A, dtype=np.uint8)
    q[:, :k] = fp8.encode(v.astype(np.float64), FMTS[fmt])
    return torch.from_numpy(q).to(d), torch.from_numpy(v.astype(np.float64)).to(d)


def filled(rows, ld, dtype, d):
    """Storage of rows of ld with one row more, holding a value no result has."""
    return torch.full((rows + 1, ld), 77.0 if dtype != torch.int8 else 77, dtype=dtype, device=d)


def untouched(t, rows, cols):
    return bool((t[:rows, cols:].float() == 77).all()) and bool((t[rows:].float() == 77).all())


class Saved:
    def __init__(self, qe, kind, rows, cols, d, pad=0):
        self.kind, self.rows, self.cols, self.h = kind, rows, cols, None
        groups = (cols + 31) // 32
        if kind == "bf16":
            self.data = filled(rows, cols + pad, torch.bfloat16, d)
            self.h = qe.make_saved(qe.SAVED_BF16, self.data, cols + pad)
        elif kind == "i8":
            self.data = filled(rows, cols + pad, torch.int8, d)
            self.exps = torch.full((rows + 1, groups + pad), 77, dtype=torch.uint8, device=d)
            self.h = qe.make_saved(qe.SAVED_I8, self.data, cols + pad, self.exps, groups + pad)

    def put(self, z):
        """Holds float32 numpy z (as the format rounds it); the values it then stands for."""
        z = np.asarray(z, dtype=np.float32)
        if self.kind == "bf16":
            self.data[:self.rows, :self.cols] = torch.from_numpy(z).to(self.data.device)
            return self.data[:self.rows, :self.cols].double()
        codes, exps = oa.pack(z)
        self.data[:self.rows, :self.cols] = torch.from_numpy(codes).to(self.data.device)
        self.exps[:self.rows, :exps.shape[1]] = torch.from_numpy(exps).to(self.data.device)
        return torch.from_numpy(oa.unpack(codes, exps)).to(self.data.device)

    def check(self, z):
        """Holds exactly z (a tensor of values exact in float32), nothing else was written."""
        if self.kind == "none":
            return
        got = self.data[:self.rows, :self.cols]
        if self.kind == "bf16":
            assert torch.equal(got, z.float().to(torch.bfloat16))
        else:
            codes, exps = oa.pack(z.float().cpu().numpy())
            assert np.array_equal(got.cpu().numpy(), codes)
            assert np.array_equal(self.exps[:self.rows, :exps.shape[1]].cpu().numpy(), exps)
            assert untouched(self.exps, self.rows, exps.shape[1])
        assert untouched(self.data, self.rows, self.cols)


def value(z, act):
    return torch.from_numpy(oa.value(z.cpu().numpy(), act)).to(z.device)


def near(got, want, tol, bf16):
    if bf16:
        tol = tol + want.abs() * (2.0 ** -8 + 2.0 ** -18)
    off = (got.double() - want).abs() - tol
    assert float(off.max()) <= 1e-37, (float(off.max()), int(off.argmax()))


def check_product(qe, d, shape, seed, act, bias, residual, out, saved, fa=0, fb=0, pad=0, in_place=False):
    m, n, k = shape
    rng = np.random.default_rng(seed)
    a, av = int_codes(rng, m, k, fa, d)
    b, bv = int_codes(rng, n, k, fb, d)
    e = -max(0, int(round(math.log2(16.0 * math.sqrt(k) / 4.0))))  # sums of about 4
    s = torch.tensor([2.0 ** (e + 5), 2.0 ** -5], dtype=torch.float32, device=d)
    z = (av @ bv.t()) * 2.0 ** e
    t = {"bf16": torch.bfloat16, "f32": torch.float32}
    q = {"bf16": qe.BF16, "f32": qe.F32, "none": qe.F32}
    bias_t = res_t = None
    if bias != "none":
        bias_t = torch.from_numpy(rng.integers(-127, 128, size=n) / 64.0).to(d).to(t[bias])
        z = z + bias_t.double()
    assert torch.equal(z, z.float().double())
    want = value(z, act)
    if residual != "none":
        res_t = filled(m, n + pad, t[residual], d)
        res_t[:m, :n] = torch.from_numpy(rng.normal(size=(m, n))).to(d)
        want = want + res_t[:m, :n].double()
    keep = Saved(qe, saved, m, n, d, pad)
    c = res_t if in_place else filled(m, n + pad, t[out], d)
    epi = qe.make_epilogue(ACT[act], bias_t, q[bias], res_t, q[residual], n + pad, keep.h)
    st = qe.qe_fp8_gemm_act(a, fa, a.shape[1], b, fb, b.shape[1], m, n, k, s[0:1], s[1:2], epi, c, q[out], n + pad)
    assert st == "OK"
    torch.cuda.synchronize()
    near(c[:m, :n], want, 16 * U * (1 + z.abs()) + 2 * U * want.abs(), out == "bf16")
    assert untouched(c, m, n)
    keep.check(z)


def check_gated(qe, d, shape, seed, act, out, saved, fa=0, fb=0, pad=0):
    m, n, k = shape
    rng = np.random.default_rng(seed)
    a, av = int_codes(rng, m, k, fa, d)
    w, wv = int_codes(rng, 2 * n, k, fb, d)
    e = -max(0, int(round(math.log2(16.0 * math.sqrt(k) / 4.0))))
    s = torch.tensor([2.0 ** (e + 5), 2.0 ** -5, 2.0 ** -6], dtype=torch.float32, device=d)
    g, u = (av @ wv[:n].t()) * 2.0 ** e, (av @ wv[n:].t()) * 2.0 ** (e - 1)
    keep = [Saved(qe, saved, m, n, d, pad) for _ in range(2)]
    t = torch.bfloat16 if out == "bf16" else torch.float32
    h = filled(m, n + pad, t, d)
    st = qe.qe_fp8_gemm_gated(a, fa, a.shape[1], w, w[n:], fb, w.shape[1], m, n, k, s[0:1], s[1:2], s[2:3], ACT[act], h,
                              qe.BF16 if out == "bf16" else qe.F32, n + pad, keep[0].h, keep[1].h)
    assert st == "OK"
    torch.cuda.synchronize()
    want = value(g, act) * u
    near(h[:m, :n], want, 16 * U * (1 + g.abs()) * u.abs() + 2 * U * want.abs(), out == "bf16")
    assert untouched(h, m, n)
    keep[0].check(g)
    keep[1].check(u)


# act, bias, residual, out, saved, fmt_a, fmt_b, pad
EPILOGUES = [("none", "none", "none", "f32", "none", 0, 0, 0), ("none", "none", "bf16", "bf16", "none", 0, 0, 0),
             ("relu", "f32", "none", "bf16", "i8", 1, 0, 1), ("gelu", "bf16", "f32", "f32", "bf16", 0, 1, 3),
             ("gelu_tanh", "f32", "bf16", "bf16", "i8", 0, 0, 16), ("silu", "bf16", "none", "f32", "i8", 1, 1, 5),
             ("silu", "none", "f32", "bf16", "bf16", 0, 0, 0)]


@pytest.mark.parametrize("epi", EPILOGUES, ids=lambda e: "-".join(map(str, e)))
@pytest.mark.parametrize("shape", SHAPES, ids=ids)
def test_product(shape, epi):
    qe, (act, bias, residual, out, saved, fa, fb, pad) = need_lib(), epi
    check_product(qe, dev(), shape, sum(shape), act, bias, residual, out, saved, fa, fb, pad)


GATES = [("silu", "bf16", "none", 0, 0, 0), ("silu", "bf16", "i8", 1, 0, 3), ("gelu", "f32", "bf16", 0, 1, 1),
         ("gelu_tanh", "bf16", "i8", 0, 0, 0), ("relu", "f32", "i8", 1, 1, 16), ("none", "bf16", "none", 0, 0, 5)]


@pytest.mark.parametrize("gate", GATES, ids=lambda e: "-".join(map(str, e)))
@pytest.mark.parametrize("shape", SHAPES, ids=ids)
def test_gated(shape, gate):
    qe, (act, out, saved, fa, fb, pad) = need_lib(), gate
    check_gated(qe, dev(), shape, sum(shape) + 1, act, out, saved, fa, fb, pad)


@pytest.mark.parametrize("tile", TILES, ids=lambda t: t[0][4:])
def test_every_small_tile(tile):
    _, gated, m, n, k = tile
    qe = need_lib()
    if gated:
        check_gated(qe, dev(), (m, n, k), 5, "silu", "bf16", "none" if m * n > 2 ** 20 else "i8")
    else:
        check_product(qe, dev(), (m, n, k), 5, "silu", "f32", "bf16", "bf16", "none" if m * n > 2 ** 20 else "i8")


@pytest.mark.parametrize("shape", [(17, 33, 1100), (50, 70, 2100), (33, 500, 4001), (112, 160, 12300), (369, 250, 12304)], ids=ids)
def test_few_blocks_of_a_long_reduction(shape):
    """Several row blocks through the kernel that splits the reduction over its waves."""
    qe, d = need_lib(), dev()
    check_product(qe, d, shape, 1, "gelu", "f32", "bf16", "bf16", "none", 0, 0, 3)
    check_product(qe, d, shape, 2, "silu", "none", "none", "f32", "i8", 1, 0, 0)
    check_gated(qe, d, shape, 3, "silu", "bf16", "none", 0, 0, 1)
    check_gated(qe, d, shape, 4, "relu", "f32", "bf16", 0, 1, 0)


@pytest.mark.parametrize("shape", [(1, 1, 1), (37, 53, 100), (256, 128, 128), (300, 520, 384), (513, 259, 1000)], ids=ids)
@pytest.mark.parametrize("tile", ["TILE_256x256", "TILE_192x256"])
def test_large_tiles(tile, shape):
    qe, d = need_lib(), dev()
    assert qe.qe_set_gemm_tile(getattr(qe, tile)) == "OK"
    try:
        check_product(qe, d, shape, 1, "gelu", "f32", "bf16", "bf16", "i8", 0, 0, 0)
        check_product(qe, d, shape, 2, "none", "none", "f32", "f32", "bf16", 1, 0, 3)
        check_gated(qe, d, shape, 3, "silu", "bf16", "i8", 0, 0, 0)
        check_gated(qe, d, shape, 4, "gelu_tanh", "f32", "bf16", 0, 1, 1)
    finally:
        assert qe.qe_set_gemm_tile(qe.TILE_AUTO) == "OK"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_residual_in_place(dtype):
    for shape in ((3, 100, 64), (200, 333, 256)):
        check_product(need_lib(), dev(), shape, 9, "silu", "none", dtype, dtype, "none", in_place=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_residual_in_place_on_large_tiles(dtype):
    qe, d = need_lib(), dev()
    assert qe.qe_set_gemm_tile(qe.TILE_256x256) == "OK"
    try:
        for shape in ((256, 256, 128), (300, 333, 256)):
            check_product(qe, d, shape, 9, "gelu", "f32", dtype, dtype, "none", in_place=True)
    finally:
        assert qe.qe_set_gemm_tile(qe.TILE_AUTO) == "OK"


def test_an_empty_reduction_leaves_bias_and_residual():
    qe, d = need_lib(), dev()
    a, bias = torch.zeros(64, dtype=torch.uint8, device=d), torch.arange(40, dtype=torch.float32, device=d)
    c, one = torch.zeros((3, 40), device=d), torch.ones(1, device=d)
    assert qe.qe_fp8_gemm_act(a, 0, 16, a, 0, 16, 3, 40, 0, one, one, qe.make_epilogue(0, bias, qe.F32), c, qe.F32, 40) == "OK"
    assert torch.equal(c, bias.expand(3, 40))


@pytest.mark.parametrize("shape", [(65, 62), (300, 520)], ids=ids)
@pytest.mark.parametrize("tile", ["TILE_AUTO", "TILE_256x256", "TILE_192x256"])
def test_an_empty_reduction_on_every_kind_of_tile(tile, shape):
    """Sums of nothing are zero: the bias through the activation, plus the residual; a gated product is zero."""
    qe, d = need_lib(), dev()
    m, n = shape
    codes, one = torch.full((max(m, n), 16), 0x3A, dtype=torch.uint8, device=d), torch.ones(1, device=d)
    bias = (torch.arange(n, device=d) - n // 2).float()
    res = torch.arange(m * n, device=d).reshape(m, n).float()
    c, h = filled(m, n, torch.float32, d), filled(m, n, torch.float32, d)
    assert qe.qe_set_gemm_tile(getattr(qe, tile)) == "OK"
    try:
        epi = qe.make_epilogue(qe.ACT_RELU, bias, qe.F32, res, qe.F32, n)
        assert qe.qe_fp8_gemm_act(codes, 0, 16, codes, 0, 16, m, n, 0, one, one, epi, c, qe.F32, n) == "OK"
        assert qe.qe_fp8_gemm_gated(codes, 0, 16, codes, codes, 0, 16, m, n, 0, one, one, one, qe.ACT_SILU, h, qe.F32, n) == "OK"
        torch.cuda.synchronize()
    finally:
        assert qe.qe_set_gemm_tile(qe.TILE_AUTO) == "OK"
    assert torch.equal(c[:m], bias.clamp(min=0) + res) and untouched(c, m, n)
    assert bool((h[:m] == 0).all()) and untouched(h, m, n)


def test_random_codes_against_float64():
    """Sums of ordinary values: the matrix instruction holds FP32 sums of 128 products, which it aligns to their
    largest before it adds (the plain GEMM's tests allow 1e-3 of the largest output)."""
    qe, d = need_lib(), dev()
    g = torch.Generator(device=d)
    g.manual_seed(4)
    x, w = torch.randn((130, 1000), generator=g, device=d), torch.randn((600, 1000), generator=g, device=d) * 0.05
    ld = rup16(1000)
    xq, wq = torch.zeros((130, ld), dtype=torch.uint8, device=d), torch.zeros((600, ld), dtype=torch.uint8, device=d)
    xq[:, :1000] = (x * 64).to(torch.float8_e4m3fn).view(torch.uint8)
    wq[:, :1000] = (w * 1024).to(torch.float8_e4m3fn).view(torch.uint8)
    xv, wv = xq[:, :1000].view(torch.float8_e4m3fn).double() / 64, wq[:, :1000].view(torch.float8_e4m3fn).double() / 1024
    s = torch.tensor([1 / 64, 1 / 1024], device=d)
    h = torch.zeros((130, 300), device=d)
    assert qe.qe_fp8_gemm_gated(xq, 0, ld, wq, wq[300:], 0, ld, 130, 300, 1000, s[0:1], s[1:2], s[1:2], qe.ACT_SILU, h, qe.F32, 300) == "OK"
    gate, up = xv @ wv[:300].t(), xv @ wv[300:].t()
    want = value(gate, "silu") * up
    assert float((h.double() - want).abs().max() / want.abs().max()) <= 1e-3


def test_nan_codes_reach_the_output_and_the_checkpoint():
    qe, d = need_lib(), dev()
    x = torch.full((3, 64), 0x38, dtype=torch.uint8, device=d)  # ones
    x[1, 7] = 0x7F
    w = torch.full((2 * 40, 64), 0x38, dtype=torch.uint8, device=d)
    one = torch.ones(1, device=d)
    keep = [Saved(qe, "i8", 3, 40, d) for _ in range(2)]
    h = torch.zeros((3, 40), device=d)
    assert qe.qe_fp8_gemm_gated(x, 0, 64, w, w[40:], 0, 64, 3, 40, 64, one, one, one, qe.ACT_RELU, h, qe.F32, 40, keep[0].h, keep[1].h) == "OK"
    assert bool(h[1].isnan().all()) and bool((h[[0, 2]] == 4096).all())
    for k in keep:
        assert k.exps[:3].tolist() == [[127, 127], [255, 255], [127, 127]] and bool((k.data[1, :40] == 0).all())


# ------------------------------------------------------------------ gradient
def check_grad(qe, d, rows, cols, seed, act, gated, kind, dtype, fmt, dense="f32", pad=0, spoil=None, accum=True, bias=None):
    rng = np.random.default_rng(seed)
    width = cols * (2 if gated else 1)
    t = {"bf16": torch.bfloat16, "f32": torch.float32}
    dd = filled(rows, cols + pad, t[dtype], d)
    dd[:rows, :cols] = torch.from_numpy(rng.normal(size=(rows, cols)) * 0.01).to(d)
    z, u = rng.normal(size=(2, rows, cols)) * 2.0
    if spoil is not None:
        spoil(dd, z)
    zs, us = Saved(qe, kind, rows, cols, d, pad), Saved(qe, kind, rows, cols, d, pad)
    zv, uv = zs.put(z), us.put(u)
    mb = meta_buffer(4, d, 2.0 ** 12)
    acc = accum_buffer(d) if accum else None
    meta = meta_of(qe, mb, fmt, 0, acc)
    q_row = torch.full((rows + 1, width + pad), 77, dtype=torch.uint8, device=d)
    q_col = torch.full((width + 1, rows + pad), 77, dtype=torch.uint8, device=d)
    snap = torch.zeros(1, device=d)
    dz = filled(rows, width + pad, t[dense], d)
    db = ws = None
    if bias is not None:
        db = torch.full((cols,), 3.0, device=d)
        ws = torch.full((-(-rows // 64) * cols + 1,), 5.0, device=d)
    st = qe.qe_act_grad(dd, {"bf16": qe.BF16, "f32": qe.F32}[dtype], cols + pad, rows, cols, ACT[act], zs.h, us.h if gated else None,
                        meta, q_row, width + pad, q_col, rows + pad, snap, dz, {"bf16": qe.BF16, "f32": qe.F32}[dense],
                        width + pad, db, qe.INIT if bias is None else bias, ws)
    assert st == "OK"
    torch.cuda.synchronize()
    assert untouched(dz, rows, width) and untouched(q_row, rows, width) and untouched(q_col, width, rows)
    got = dz[:rows, :width]
    ddv = dd[:rows, :cols].double()
    slope = torch.from_numpy(oa.slope(zv.cpu().numpy(), act)).to(d)
    want = ddv * slope * uv if gated else ddv * slope
    tol = (16 + 4 * zv.abs()) * U * (ddv * uv if gated else ddv).abs()
    if gated:
        want = torch.cat((want, ddv * value(zv, act)), 1)
        tol = torch.cat((tol, 16 * U * (1 + zv.abs()) * ddv.abs()), 1)
    fine = want.isfinite()
    assert torch.equal(fine, got.isfinite())
    near(torch.where(fine, got.double(), 0.0), torch.where(fine, want, 0.0), torch.where(fine, tol + 2 * U * want.abs(), 0.0), dense == "bf16")
    codes = q_row[:rows, :width]
    assert torch.equal(q_col[:width, :rows], codes.t())
    assert float(snap) == 2.0 ** -12
    top = accum_value(acc) if accum else float(mb[0])
    if dense == "f32":  # the values that were encoded
        assert np.array_equal(codes.cpu().numpy(), fp8.encode(got.double().cpu().numpy() * 2.0 ** 12, FMTS[fmt]))
        peak = float(got.abs().max()) if bool(fine.all()) else math.nan if bool(got.isnan().any()) else math.inf
        assert top == peak or (math.isnan(top) and math.isnan(peak))
        if bias is not None:
            total = got.double().sum(0) + (3.0 if bias == qe.ACCUM else 0.0)
            assert bool(((db.double() - total).abs() <= (rows + 8) * U * (got.double().abs().sum(0) + 3.0)).all())
            assert float(ws[-1]) == 5.0
    return db


GRAD_SHAPES = [(1, 1), (1, 32), (2, 33), (17, 127), (64, 128), (65, 200), (130, 257), (300, 300)]
# act, gated, saved, dd, format, dense, pad, accumulator
GRADS = [("silu", True, "i8", "bf16", 1, "f32", 0, True), ("silu", True, "i8", "f32", 0, "bf16", 3, True),
         ("gelu_tanh", True, "bf16", "bf16", 1, "f32", 1, False), ("gelu", False, "i8", "f32", 1, "f32", 3, True),
         ("gelu_tanh", False, "i8", "bf16", 0, "f32", 0, False), ("relu", False, "bf16", "f32", 1, "f32", 16, True),
         ("none", True, "bf16", "f32", 0, "f32", 5, True), ("gelu", True, "i8", "bf16", 0, "f32", 0, True)]


@pytest.mark.parametrize("g", GRADS, ids=lambda g: "-".join(map(str, g)))
@pytest.mark.parametrize("shape", GRAD_SHAPES, ids=ids)
def test_grad(shape, g):
    act, gated, kind, dtype, fmt, dense, pad, accum = g
    check_grad(need_lib(), dev(), *shape, sum(shape), act, gated, kind, dtype, fmt, dense, pad, accum=accum)


@pytest.mark.parametrize("shape", GRAD_SHAPES, ids=ids)
def test_bias_grad(shape):
    qe, d = need_lib(), dev()
    for mode in (qe.INIT, qe.ACCUM):
        a = check_grad(qe, d, *shape, 3, "silu", False, "i8", "bf16", 1, bias=mode)
        b = check_grad(qe, d, *shape, 3, "silu", False, "i8", "bf16", 1, bias=mode)
        assert torch.equal(a, b)


@pytest.mark.parametrize("gated", [False, True])
def test_grad_of_large_tensors(gated):
    """Hundreds of 64-row tiles, in more than one group of row tiles."""
    check_grad(need_lib(), dev(), 2900, 3001, 8, "gelu_tanh", gated, "bf16", "bf16", 1, bias=None if gated else need_lib().INIT)


@pytest.mark.parametrize("gated,rows,cols", [(False, 4200, 4300), (True, 8300, 2100)])
def test_grad_of_tall_tiles(gated, rows, cols):
    """Past 1024 tiles of 128 rows, where the tiles have 128 rows."""
    check_grad(need_lib(), dev(), rows, cols, 8, "silu", gated, "bf16", "bf16", 1, bias=None if gated else need_lib().INIT)


def test_grad_of_infinities_and_nans():
    """A NaN gradient, an infinite one and a pre-activation that is not finite: NaN for the whole saved group."""
    qe, d = need_lib(), dev()

    def spoil(dd, z):
        dd[0, 3], dd[40, 70], z[9, 64] = math.nan, math.inf, math.nan
    for gated in (False, True):
        check_grad(qe, d, 65, 100, 2, "silu", gated, "i8", "f32", 1, spoil=spoil)


def test_grad_of_nothing():
    qe, d = need_lib(), dev()
    snap, db = torch.zeros(1, device=d), torch.ones(7, device=d)
    mb = meta_buffer(4, d, 8.0)
    z = qe.make_saved(qe.SAVED_I8, 0, 7, 0, 1)
    ws = torch.ones(7, device=d)
    assert qe.qe_act_grad(0, qe.BF16, 7, 0, 7, 4, z, None, meta_of(qe, mb, 0), scale_inv_snapshot=snap, dbias=db, workspace=ws) == "OK"
    assert float(snap) == 0.125 and bool((db == 0).all()) and bool((ws == 1).all())
    assert qe.qe_act_grad(0, qe.BF16, 0, 5, 0, 4, z) == "OK"


@pytest.mark.parametrize("act", [a for a in oa.ACTS if a != "relu"])
def test_gradient_is_the_difference_quotient_of_the_forward(act):
    """dD/dbias of the product, by differences of the forward and by qe_act_grad on what the forward saved.

    h = 1/16: truncation h^2/6 |f'''| with |f'''| <= 2 for these, 1.4e-3; FP32 noise 16 u 8 / h; and the saved z
    is the forward's own in BF16, off by 2^-8 |z| |f''| with |f''| <= 1.2 and |z f''| < 1.2 (gelu: z phi (2 - z^2))."""
    qe, d = need_lib(), dev()
    rng = np.random.default_rng(6)
    m, n, k = 33, 70, 100
    a, _ = int_codes(rng, m, k, 0, d)
    b, _ = int_codes(rng, n, k, 0, d)
    s = torch.tensor([2.0 ** -6, 1.0], device=d)
    bias = torch.from_numpy(rng.integers(-64, 65, size=n) / 32.0).float().to(d)
    keep = Saved(qe, "bf16", m, n, d)
    got = []
    for step in (1 / 16, -1 / 16, 0.0):
        c, moved = torch.zeros((m, n), device=d), bias + step
        epi = qe.make_epilogue(ACT[act], moved, qe.F32, saved=keep.h)
        assert qe.qe_fp8_gemm_act(a, 0, a.shape[1], b, 0, b.shape[1], m, n, k, s[0:1], s[1:2], epi, c, qe.F32, n) == "OK"
        got.append(c.double())
    dz, dd = torch.zeros((m, n), device=d), torch.ones((m, n), device=d)
    assert qe.qe_act_grad(dd, qe.F32, n, m, n, ACT[act], keep.h, dz=dz, ld_dz=n) == "OK"
    off = float((dz.double() - (got[0] - got[1]) * 8).abs().max())
    assert off <= 1.4e-3 + 2e-4 + 2.0 ** -8 * 1.2


# ------------------------------------------------------------------ checkpoints
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape,pad", [((1, 1), 0), ((1, 31), 1), ((3, 32), 0), ((5, 33), 2), ((64, 128), 0), ((65, 129), 7), ((200, 300), 4)], ids=str)
def test_save_and_restore(shape, pad, dtype):
    qe, d = need_lib(), dev()
    rows, cols = shape
    rng = np.random.default_rng(rows + cols)
    t, q = {"bf16": (torch.bfloat16, qe.BF16), "f32": (torch.float32, qe.F32)}[dtype]
    v = rng.normal(size=shape) * 10.0 ** rng.integers(-40, 38, size=(rows, 1))
    if cols > 1:
        v[0, 1] = math.inf
    v[rows // 2, cols // 2] = math.nan
    if rows > 3:
        v[2, :], v[3, :] = 0.0, 1e-45
    x = filled(rows, cols + pad, t, d)
    x[:rows, :cols] = torch.from_numpy(v.astype(np.float32)).to(d)
    keep = Saved(qe, "i8", rows, cols, d, pad)
    assert qe.qe_act_save(x, q, cols + pad, rows, cols, keep.h) == "OK"
    torch.cuda.synchronize()
    keep.check(x[:rows, :cols])
    want = oa.unpack(*oa.pack(x[:rows, :cols].float().cpu().numpy()))
    for ot, oq in ((torch.bfloat16, qe.BF16), (torch.float32, qe.F32)):
        y = filled(rows, cols + pad, ot, d)
        assert qe.qe_act_restore(keep.h, rows, cols, y, oq, cols + pad) == "OK"
        torch.cuda.synchronize()
        assert np.array_equal(y[:rows, :cols].double().cpu().numpy(), want, equal_nan=True)
        assert untouched(y, rows, cols)


def test_offsets_past_32_bits():
    """Rows 4 MiB (codes) and 2^23 elements (checkpoints) apart, over 4 GiB of each."""
    qe, d = need_lib(), dev()
    rows, ld = 1040, 1 << 22
    a = torch.zeros((rows, ld), dtype=torch.uint8, device=d)
    a[:, :16] = torch.randint(0x30, 0x40, (rows, 16), dtype=torch.uint8, device=d)
    b = torch.randint(0x30, 0x40, (40, 16), dtype=torch.uint8, device=d)
    one, c, c2 = torch.ones(1, device=d), torch.zeros((rows, 40), device=d), torch.zeros((rows, 40), device=d)
    assert qe.qe_fp8_gemm_act(a, 0, ld, b, 0, 16, rows, 40, 16, one, one, None, c, qe.F32, 40) == "OK"
    near_a = a[:, :16].contiguous()
    assert qe.qe_fp8_gemm_act(near_a, 0, 16, b, 0, 16, rows, 40, 16, one, one, None, c2, qe.F32, 40) == "OK"
    assert torch.equal(c, c2) and float(c.abs().min()) > 0
    assert qe.qe_fp8_gemm_act(b, 0, 16, a, 0, ld, 40, rows, 16, one, one, None, c2.view(40, rows), qe.F32, rows) == "OK"
    assert torch.equal(c2.view(40, rows).t(), c)
    del a
    x, far = torch.randn((520, 64), device=d), torch.zeros((520, 1 << 23), dtype=torch.int8, device=d)
    exps, y = torch.zeros((520, 2), dtype=torch.uint8, device=d), torch.zeros((520, 64), device=d)
    s = qe.make_saved(qe.SAVED_I8, far, 1 << 23, exps, 2)
    assert qe.qe_act_save(x, qe.F32, 64, 520, 64, s) == "OK" and qe.qe_act_restore(s, 520, 64, y, qe.F32, 64) == "OK"
    assert np.array_equal(y.cpu().numpy(), oa.unpack(*oa.pack(x.cpu().numpy())))
    dz = torch.zeros((520, 64), device=d)
    assert qe.qe_act_grad(torch.ones((520, 64), device=d), qe.F32, 64, 520, 64, qe.ACT_RELU, s, dz=dz, ld_dz=64) == "OK"
    assert torch.equal(dz, (y > 0).float())


# ------------------------------------------------------------------ streams and graphs
def test_side_stream_and_graph_replay():
    """The whole feed-forward, forward and backward, captured by the caller: every replay equals the eager pass on
    the same inputs, with other work between the replays."""
    qe, d = need_lib(), dev()
    m, f, k = 70, 96, 160
    rng = np.random.default_rng(2)
    w, _ = int_codes(rng, 2 * f, k, 0, d)
    xs = [int_codes(rng, m, k, 0, d)[0] for _ in range(3)]
    s = torch.tensor([2.0 ** -5, 1.0], device=d)
    x = xs[0].clone()
    keep = [Saved(qe, "i8", m, f, d) for _ in range(2)]
    h, dh, dz = torch.zeros((m, f), device=d), torch.randn((m, f), device=d), torch.zeros((m, 2 * f), device=d)
    db, ws = torch.zeros(f, device=d), torch.zeros(2 * f, device=d)

    def step(stream):
        assert qe.qe_fp8_gemm_gated(x, 0, x.shape[1], w, w[f:], 0, w.shape[1], m, f, k, s[0:1], s[1:2], s[1:2], qe.ACT_SILU, h,
                                    qe.F32, f, keep[0].h, keep[1].h, stream=stream) == "OK"
        assert qe.qe_act_grad(dh, qe.F32, f, m, f, qe.ACT_SILU, keep[0].h, keep[1].h, dz=dz, ld_dz=2 * f, stream=stream) == "OK"
        assert qe.qe_act_grad(dh, qe.F32, f, m, f, qe.ACT_SILU, keep[0].h, dbias=db, workspace=ws, stream=stream) == "OK"
    side, want = torch.cuda.Stream(), []
    for v in xs:
        x.copy_(v)
        side.wait_stream(torch.cuda.current_stream())
        step(side)
        torch.cuda.current_stream().wait_stream(side)
        want.append([t.clone() for t in (h, dz, db)])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(torch.cuda.current_stream())
    for i in (1, 0, 2, 2, 1):
        x.copy_(xs[i])
        for t in (h, dz, db):
            t.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((h, dz, db), want[i]))
        torch.randn(1000, device=d).sort()
