"""FP8 casts and products with a scale for each block of 128 on the GPU, against float64.

Casts are exact: codes and exponent bytes have to be the oracle's.  Products read codes of small integers at scales
2^-1 .. 2^1, so every sum is a multiple of 2^-2 below 2^22 and exact in FP32; with u = 2^-24 an output may then be off by
its activation and roundings, 16 u (1 + |z|), as for the products with one scale, and by half an ulp of BF16, 2^-8.
"""
import numpy as np
import pytest

from oracle import blocks as ob
from oracle import fp8
from tests.act_tiles import TILES
from tests.gpu_util import dev, torch
from tests.libqe import need_lib
from tests.test_gpu_activation import ACT, FMTS, Saved, U, filled, near, untouched, value

pytestmark = pytest.mark.gpu
T = {"bf16": torch.bfloat16, "f32": torch.float32}
ids = lambda s: "x".join(map(str, s)) if isinstance(s, tuple) else None  # noqa: E731


def dtype(qe, t):
    return qe.BF16 if t == torch.bfloat16 else qe.F32


def matrix(qe, t):
    return None if t is None else qe.make_matrix(t, t.stride(0), dtype(qe, t.dtype))


class Blocks:
    """Storage for [rows, cols] codes and their bytes, with a row more and `pad` columns that hold 77."""

    def __init__(self, qe, rows, cols, fmt, block_rows, d, pad=0):
        self.rows, self.cols, self.fmt, self.br = rows, cols, fmt, block_rows
        self.groups = (-(-rows // block_rows), -(-cols // 128))
        self.q = torch.full((rows + 1, cols + pad), 77, dtype=torch.uint8, device=d)
        self.e = torch.full((self.groups[0] + 1, self.groups[1] + pad), 77, dtype=torch.uint8, device=d)
        self.h = qe.make_blocked(self.q, cols + pad, self.e, self.groups[1] + pad, fmt, block_rows)

    def get(self):
        return self.q[:self.rows, :self.cols].cpu().numpy(), self.e[:self.groups[0], :self.groups[1]].cpu().numpy()

    def check(self, x):
        codes, exps = ob.pack(x, FMTS[self.fmt], self.br)
        q, e = self.get()
        assert np.array_equal(e, exps)
        nan = np.isnan(fp8.decode(codes, FMTS[self.fmt]))
        assert np.array_equal(np.isnan(fp8.decode(q, FMTS[self.fmt])), nan)
        assert np.array_equal(q[~nan], codes[~nan])
        assert untouched(self.q, self.rows, self.cols) and untouched(self.e, *self.groups)


def check_cast(qe, d, x, fmt, block_rows, row=True, col=True, pad=0, t="f32"):
    """x: float numpy values."""
    rows, cols = x.shape
    inp = filled(rows, cols + pad, T[t], d)
    inp[:rows, :cols] = torch.from_numpy(x).to(d)
    r, c = Blocks(qe, rows, cols, fmt, block_rows, d, pad), Blocks(qe, cols, rows, fmt, block_rows, d, pad)
    st = qe.qe_quantize_fp8_block(qe.make_matrix(inp, cols + pad, dtype(qe, T[t])), rows, cols, r.h if row else None, c.h if col else None)
    assert st == "OK"
    torch.cuda.synchronize()
    v = inp[:rows, :cols].double().cpu().numpy()
    if row:
        r.check(v)
    if col:
        c.check(v.T)
    return r, c


CAST_SHAPES = [(1, 1), (1, 128), (256, 384), (131, 512), (1, 513), (3, 130), (127, 129), (128, 128), (129, 255), (250, 300), (16, 1000), (300, 7)]


@pytest.mark.parametrize("how", [("f32", 0, 1, 0), ("bf16", 0, 1, 0), ("bf16", 1, 1, 3), ("f32", 1, 1, 1), ("bf16", 0, 128, 0), ("f32", 1, 128, 5)],
                         ids=lambda h: "-".join(map(str, h)))
@pytest.mark.parametrize("shape", CAST_SHAPES, ids=ids)
def test_cast(shape, how):
    t, fmt, block_rows, pad = how
    rng = np.random.default_rng(sum(shape))
    x = rng.normal(size=shape) * np.exp(2.0 * rng.normal(size=(shape[0], 1)))
    check_cast(need_lib(), dev(), x, fmt, block_rows, pad=pad, t=t)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_cast_one_order(block_rows):
    x = np.random.default_rng(2).normal(size=(200, 333))
    for row, col in ((True, False), (False, True)):
        check_cast(need_lib(), dev(), x, 0, block_rows, row, col, pad=1)


@pytest.mark.parametrize("fmt", [0, 1], ids=FMTS)
@pytest.mark.parametrize("block_rows", [1, 128])
def test_cast_of_special_values(block_rows, fmt):
    """Zeros of both signs, subnormal and largest values, amaxes on both sides of fmax's mantissa; infinities and NaN spoil their block alone."""
    rng = np.random.default_rng(3)
    x = rng.normal(size=(260, 390)).astype(np.float32)
    x[0, :128], x[1, :128] = 0.0, -0.0
    x[2, :128] = 1e-40
    x[3, :128], x[3, 5] = 1e-44, -2.0 ** -149
    x[4, 130] = 3.4028235e38
    x[5, 130] = -np.float32(1.75 * 2.0 ** 127)
    for i, a in enumerate((448.0, 448.00003, 57344.0, 57344.004, 1.75, np.nextafter(np.float32(1.75), np.float32(2)), 2.0 ** -126)):
        x[8 + i, 256:384] = a * rng.uniform(-1, 1, size=128).astype(np.float32)
        x[8 + i, 300] = a
    x[20, 40], x[21, 200], x[22, 389], x[259, 3] = np.nan, np.inf, -np.inf, np.nan
    check_cast(need_lib(), dev(), x, fmt, block_rows)


def test_cast_of_long_offsets():
    """Elements past 2^31 (BF16, 4.3 GB): sampled rows and columns against the oracle, every transposed block of them."""
    qe, d = need_lib(), dev()
    rows, cols = 65_613, 32_808
    g = torch.Generator(device=d)
    g.manual_seed(1)
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device=d)
    for r in range(0, rows, 8192):
        x[r:r + 8192].normal_(generator=g)
    q, e = torch.zeros((rows, cols), dtype=torch.uint8, device=d), torch.zeros((rows, 257), dtype=torch.uint8, device=d)
    qt, et = torch.zeros((cols, rows), dtype=torch.uint8, device=d), torch.zeros((cols, 513), dtype=torch.uint8, device=d)
    assert qe.qe_quantize_fp8_block(matrix(qe, x), rows, cols, qe.make_blocked(q, cols, e, 257, 0), qe.make_blocked(qt, rows, et, 513, 0)) == "OK"
    for r in (0, 127, 40_000, 65_471, 65_472, rows - 1):
        codes, exps = ob.pack(x[r:r + 1].double().cpu().numpy(), "E4M3")
        assert np.array_equal(q[r:r + 1].cpu().numpy(), codes) and np.array_equal(e[r:r + 1].cpu().numpy(), exps), r
    for c in (0, 128, 20_000, 32_767, cols - 1):
        codes, exps = ob.pack(x[:, c:c + 1].double().cpu().numpy().T, "E4M3")
        assert np.array_equal(qt[c:c + 1].cpu().numpy(), codes) and np.array_equal(et[c:c + 1].cpu().numpy(), exps), c


# ------------------------------------------------------------------ products
def operand(qe, rng, rows, k, fmt, block_rows, d, exps=None):
    """Codes of integers in -6 .. 6 at scales 2^-1 .. 2^1 (other codes and bytes behind the last column and block), their values, the handle."""
    ld, groups, lde = -(-k // 16) * 16, -(-k // 128), -(-k // 512) * 4
    v = rng.integers(-6, 7, size=(rows, k)).astype(np.float64)
    q = np.full((rows, max(ld, 16)), 0x3A, dtype=np.uint8)
    q[:, :k] = fp8.encode(v, FMTS[fmt])
    e = np.full((-(-rows // block_rows), max(lde, 4)), 200, dtype=np.uint8)
    e[:, :groups] = rng.integers(126, 129, size=(e.shape[0], groups)) if exps is None else exps
    v = ob.unpack(q[:, :k], e[:, :groups], FMTS[fmt], block_rows)
    q, e = torch.from_numpy(q).to(d), torch.from_numpy(e).to(d)
    return q, e, torch.from_numpy(v).to(d), qe.make_blocked(q, q.shape[1], e, e.shape[1], fmt, block_rows)


def check_product(qe, d, shape, seed, out="bf16", fa=0, fb=0, ba=1, bb=128, act="none", bias="none", residual="none", saved="none", pad=0,
                  in_place=False):
    m, n, k = shape
    rng = np.random.default_rng(seed)
    qa, ea, av, ha = operand(qe, rng, m, k, fa, ba, d)
    qb, eb, bv, hb = operand(qe, rng, n, k, fb, bb, d)
    z = av @ bv.t()
    q = {"bf16": qe.BF16, "f32": qe.F32, "none": qe.F32}
    bias_t = res_t = None
    if bias != "none":
        bias_t = torch.from_numpy(rng.integers(-127, 128, size=n) / 4.0).to(d).to(T[bias])
        z = z + bias_t.double()
    assert torch.equal(z, z.float().double())
    want = value(z, act)
    if residual != "none":
        res_t = filled(m, n + pad, T[residual], d)
        res_t[:m, :n] = torch.from_numpy(rng.normal(size=(m, n))).to(d)
        want = want + res_t[:m, :n].double()
    keep = Saved(qe, saved, m, n, d, pad)
    c = res_t if in_place else filled(m, n + pad, T[out], d)
    epi = qe.make_epilogue(ACT[act], bias_t, q[bias], res_t, q[residual], n + pad, keep.h)
    assert qe.qe_fp8_gemm_block(ha, hb, m, n, k, epi, c, q[out], n + pad) == "OK"
    torch.cuda.synchronize()
    near(c[:m, :n], want, 16 * U * (1 + z.abs()) * (act != "none") + 2 * U * want.abs() * (residual != "none"), out == "bf16")
    assert untouched(c, m, n)
    keep.check(z)
    del qa, qb, ea, eb


SHAPES = [(1, 1, 1), (1, 32, 16), (2, 33, 100), (16, 64, 128), (17, 130, 257), (37, 53, 100), (64, 64, 512), (65, 200, 130), (128, 256, 256),
          (255, 511, 129), (300, 520, 384), (1, 300, 1500), (5, 96, 4100), (513, 257, 1000), (130, 70, 2600)]
HOW = [dict(out="f32"), dict(fa=1, pad=3), dict(bb=1, fa=1, out="f32", residual="f32", in_place=True), dict(ba=128, bb=1, fb=1, bias="f32", act="relu"),
       dict(ba=128, bb=128, act="silu", saved="i8", residual="bf16", pad=1), dict(fb=1, fa=1, act="gelu", bias="bf16", saved="bf16", out="f32")]


@pytest.mark.parametrize("how", HOW, ids=lambda h: "-".join(f"{k}{v}" for k, v in h.items()))
@pytest.mark.parametrize("shape", SHAPES, ids=ids)
def test_product(shape, how):
    check_product(need_lib(), dev(), shape, sum(shape), **how)


@pytest.mark.parametrize("shape", [(17, 33, 1100), (50, 70, 2100), (33, 500, 4001), (112, 160, 12300), (369, 250, 12304), (16, 4096, 2050)], ids=ids)
def test_few_blocks_of_a_long_reduction(shape):
    qe, d = need_lib(), dev()
    check_product(qe, d, shape, 1, act="gelu", bias="f32", residual="bf16", pad=3)
    check_product(qe, d, shape, 2, out="f32", bb=1, fa=1, saved="i8", act="silu")


@pytest.mark.parametrize("tile", [t for t in TILES if not t[1]], ids=lambda t: t[0][4:])
def test_every_small_tile(tile):
    """Products that the tile choice gives to each kernel; with 10 and 11 K tiles, three groups of scales, the last one short."""
    _, _, m, n, k = tile
    qe, d = need_lib(), dev()
    saved = "none" if m * n > 2 ** 20 else "i8"
    check_product(qe, d, (m, n, k), 5, act="silu", bias="f32", residual="bf16", saved=saved)
    check_product(qe, d, (m, n, k + 700), 6, bb=1, fa=1, out="f32")


@pytest.mark.parametrize("shape", [(1, 1, 1), (37, 53, 100), (256, 128, 128), (300, 520, 384), (513, 259, 1000), (260, 270, 4100), (192, 256, 640)], ids=ids)
@pytest.mark.parametrize("tile", ["TILE_256x256", "TILE_192x256"])
def test_large_tiles(tile, shape):
    qe, d = need_lib(), dev()
    assert qe.qe_set_gemm_tile(getattr(qe, tile)) == "OK"
    try:
        check_product(qe, d, shape, 1, act="gelu", bias="f32", residual="bf16", saved="i8")
        check_product(qe, d, shape, 2, bb=1, fa=1, out="f32", residual="f32", in_place=True, pad=3)
        check_product(qe, d, shape, 3, ba=128, bb=1, fb=1)
    finally:
        assert qe.qe_set_gemm_tile(qe.TILE_AUTO) == "OK"


@pytest.mark.parametrize("tile", ["TILE_256x256", "TILE_192x256"])
@pytest.mark.parametrize("out,residual", [("bf16", "none"), ("bf16", "bf16"), ("f32", "none"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
def test_bare_sums_of_large_tiles(tile, out, residual):
    """Whole tiles of sums with at most a residual of their type, in place and apart, beside tiles at the edges; odd rows."""
    qe, d = need_lib(), dev()
    assert qe.qe_set_gemm_tile(getattr(qe, tile)) == "OK"
    try:
        for shape, pad in (((520, 516, 300), 0), ((520, 516, 1100), 4), ((260, 513, 129), 2)):
            check_product(qe, d, shape, 4, out=out, residual=residual, bb=1, pad=pad)
            if residual == out:
                check_product(qe, d, shape, 5, out=out, residual=residual, fa=1, pad=pad, in_place=True)
    finally:
        assert qe.qe_set_gemm_tile(qe.TILE_AUTO) == "OK"


@pytest.mark.parametrize("m,tile", [(3, "TILE_AUTO"), (130, "TILE_AUTO"), (520, "TILE_256x256"), (520, "TILE_192x256")])
def test_products_of_long_strides(m, tile):
    """Rows as far apart as they may be, outputs and residuals past 2^31 elements: the bits of the same call on packed rows."""
    qe, d = need_lib(), dev()
    rng = np.random.default_rng(3)
    n, k, ld = 512, 384, 2 ** 23 - 16
    qa, ea, _, ha = operand(qe, rng, m, k, 0, 1, d)
    qb, eb, _, hb = operand(qe, rng, n, k, 1, 128, d)
    wide = []
    for q, e, br, fmt in ((qa, ea, 1, 0), (qb, eb, 128, 1)):
        t = torch.empty((q.shape[0], ld), dtype=torch.uint8, device=d)
        t[:, :k] = q[:, :k]
        wide.append((t, qe.make_blocked(t, ld, e, e.shape[1], fmt, br)))
    assert qe.qe_set_gemm_tile(getattr(qe, tile)) == "OK"
    try:
        for ldc in (2 ** 22, 2 ** 23 + 8):  # 2^22: whole tiles of bare sums, 128 rows of which stay below 2^31 bytes
            res = torch.from_numpy(rng.normal(size=(m, n))).to(d).bfloat16()
            c, far, far_res = torch.zeros((m, n), dtype=torch.bfloat16, device=d), *(torch.empty((m, ldc), dtype=torch.bfloat16, device=d) for _ in range(2))
            far_res[:, :n], far[:, n:n + 8] = res, 3.0
            assert qe.qe_fp8_gemm_block(ha, hb, m, n, k, qe.make_epilogue(residual=res, residual_dtype=qe.BF16, ld_residual=n), c, qe.BF16, n) == "OK"
            assert qe.qe_fp8_gemm_block(wide[0][1], wide[1][1], m, n, k, qe.make_epilogue(residual=far_res, residual_dtype=qe.BF16, ld_residual=ldc),
                                        far, qe.BF16, ldc) == "OK"
            assert torch.equal(far[:, :n], c) and bool((far[:, n:n + 8] == 3).all())
            del far, far_res
    finally:
        assert qe.qe_set_gemm_tile(qe.TILE_AUTO) == "OK"


def test_random_codes_against_float64():
    """Ordinary values: FP32 sums of 128 products which the instruction aligns to their largest; the plain product's tests allow 1e-3 of the largest."""
    qe, d = need_lib(), dev()
    rng = np.random.default_rng(6)
    m, n, k = 300, 520, 1100
    x, w = rng.normal(size=(m, k)) * np.exp(rng.normal(size=(m, 1))), rng.normal(size=(n, k)) * 0.05
    ops = []
    for v, br in ((x, 1), (w, 128)):
        codes, exps = ob.pack(v, "E4M3", br)
        q, e = np.zeros((v.shape[0], 1104), np.uint8), np.zeros((exps.shape[0], 12), np.uint8)
        q[:, :k], e[:, :exps.shape[1]] = codes, exps
        ops.append((torch.from_numpy(q).to(d), torch.from_numpy(e).to(d), ob.unpack(codes, exps, "E4M3", br)))
    c = torch.zeros((m, n), device=d)
    h = [qe.make_blocked(q, 1104, e, 12, 0, br) for (q, e, _), br in zip(ops, (1, 128))]
    assert qe.qe_fp8_gemm_block(h[0], h[1], m, n, k, None, c, qe.F32, n) == "OK"
    want = ops[0][2] @ ops[1][2].T
    assert np.abs(c.cpu().numpy() - want).max() / np.abs(want).max() <= 1e-3


@pytest.mark.parametrize("shape", [(3, 40, 700), (130, 70, 700), (600, 520, 700)], ids=ids)
def test_scales_of_every_size(shape):
    """Bytes far apart: 2^-126 by 2^126 and back give ordinary sums; 255 is NaN, for its rows alone."""
    qe, d = need_lib(), dev()
    m, n, k = shape
    rng = np.random.default_rng(7)
    for ea, eb in ((1, 253), (253, 1), (127 - 60, 127 + 64), (254, 0)):
        *held, av, ha = operand(qe, rng, m, k, 0, 1, d, ea)
        *held_b, bv, hb = operand(qe, rng, n, k, 0, 128, d, eb)
        c = torch.zeros((m, n), device=d)
        assert qe.qe_fp8_gemm_block(ha, hb, m, n, k, None, c, qe.F32, n) == "OK"
        assert torch.equal(c.double(), av @ bv.t()), (ea, eb)
    q, e, av, ha = operand(qe, rng, m, k, 0, 1, d)
    *held, bv, hb = operand(qe, rng, n, k, 0, 128, d)
    e[m - 1, 2] = 255
    c = torch.zeros((m, n), device=d)
    assert qe.qe_fp8_gemm_block(ha, hb, m, n, k, None, c, qe.F32, n) == "OK"
    assert bool(c[m - 1].isnan().all()) and torch.equal(c[:m - 1].double(), (av @ bv.t())[:m - 1])


def test_nan_blocks_reach_the_output():
    """What the cast makes of a NaN or an infinity shows in every output that its block reaches."""
    qe, d = need_lib(), dev()
    x = torch.ones((3, 256), device=d)
    x[1, 200], x[2, 3] = float("inf"), float("nan")
    w = torch.ones((40, 256), device=d)
    ops = []
    for t, br in ((x, 1), (w, 128)):
        q, e = torch.zeros(t.shape, dtype=torch.uint8, device=d), torch.zeros((t.shape[0], 4), dtype=torch.uint8, device=d)
        ops.append((qe.make_blocked(q, 256, e, 4, 0, br), q, e))
        assert qe.qe_quantize_fp8_block(matrix(qe, t), t.shape[0], 256, ops[-1][0]) == "OK"
    c = torch.zeros((3, 40), device=d)
    assert qe.qe_fp8_gemm_block(ops[0][0], ops[1][0], 3, 40, 256, None, c, qe.F32, 40) == "OK"
    assert bool((c[0] == 256).all()) and bool(c[1:].isnan().all())


@pytest.mark.parametrize("shape", [(3, 40), (300, 520)], ids=ids)
def test_an_empty_reduction_leaves_bias_and_residual(shape):
    qe, d = need_lib(), dev()
    m, n = shape
    q, e = torch.full((max(shape), 16), 0x3A, dtype=torch.uint8, device=d), torch.full((max(shape), 4), 255, dtype=torch.uint8, device=d)
    h = qe.make_blocked(q, 16, e, 4, 0)
    bias, res = torch.arange(n, dtype=torch.float32, device=d), torch.ones((m, n), device=d)
    c = filled(m, n, torch.float32, d)
    assert qe.qe_fp8_gemm_block(h, h, m, n, 0, qe.make_epilogue(0, bias, qe.F32, res, qe.F32, n), c, qe.F32, n) == "OK"
    torch.cuda.synchronize()
    assert torch.equal(c[:m], (bias + 1).expand(m, n)) and untouched(c, m, n)


def test_two_streams_and_a_replayed_graph():
    """Cast, product and accumulation captured on one stream and replayed between eager calls on another: every replay equals the eager result."""
    qe, d = need_lib(), dev()
    m, n, k = 200, 264, 640
    g = torch.Generator(device=d)
    g.manual_seed(8)
    x, w = torch.randn((m, k), generator=g, device=d), torch.randn((n, k), generator=g, device=d)
    xq, xe = torch.zeros((m, k), dtype=torch.uint8, device=d), torch.zeros((m, 8), dtype=torch.uint8, device=d)
    wq, we = torch.zeros((n, k), dtype=torch.uint8, device=d), torch.zeros((3, 8), dtype=torch.uint8, device=d)
    hx, hw = qe.make_blocked(xq, k, xe, 8, 0), qe.make_blocked(wq, k, we, 8, 0, 128)
    c = torch.zeros((m, n), device=d)

    def step():
        assert qe.qe_quantize_fp8_block(matrix(qe, x), m, k, hx) == "OK"
        assert qe.qe_quantize_fp8_block(matrix(qe, w), n, k, hw) == "OK"
        assert qe.qe_fp8_gemm_block(hx, hw, m, n, k, None, c, qe.F32, n) == "OK"
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        x.mul_(-1.5)
        c.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = c.clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.synchronize()
        assert torch.equal(got, c) and float(c.abs().max()) > 0
