"""What block scales add to a product's arithmetic: nothing.  The matrix instruction applies powers of two to its products, so
the sums have the bits of the product with one scale per operand, at equal scales and where the operands' scales cancel."""
import pytest

from tests.gpu_util import dev, torch
from tests.libqe import need_lib

pytestmark = pytest.mark.gpu

# 16 rows or fewer on a tile: by themselves they split the reduction over waves, with block scales in another order
SHAPES = [(130, 200, 128, "TILE_AUTO"), (300, 520, 1000, "TILE_AUTO"), (520, 300, 4100, "TILE_256x256"), (520, 300, 4100, "TILE_192x256"),
          (7, 300, 1500, "TILE_256x256")]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("fa,fb", [(0, 0), (1, 0), (0, 1), (1, 1)])
def test_sums_are_those_of_one_scale(shape, fa, fb):
    qe, d = need_lib(), dev()
    m, n, k, tile = shape
    g = torch.Generator(device=d)
    g.manual_seed(m + k)
    types = (torch.float8_e4m3fn, torch.float8_e5m2)
    ld, groups, lde = -(-k // 16) * 16, -(-k // 128), -(-k // 512) * 4
    codes, exps = [], []
    for rows, fmt, step in ((m, fa, 1), (n, fb, 128)):
        x = torch.randn((rows, ld), generator=g, device=d) * 8
        x[:, ::97] *= 10  # |x| stays far below fmax
        codes.append(x.to(types[fmt]))
        exps.append(torch.full((-(-rows // step), lde), 127, dtype=torch.uint8, device=d))
    one = torch.ones(1, device=d)
    c = [torch.zeros((m, n), device=d) for _ in range(3)]
    assert qe.qe_set_gemm_tile(getattr(qe, tile)) == "OK"
    try:
        assert qe.qe_fp8_gemm_act(codes[0], fa, ld, codes[1], fb, ld, m, n, k, one, one, None, c[0], qe.F32, n) == "OK"
        a, b = qe.make_blocked(codes[0], ld, exps[0], lde, fa), qe.make_blocked(codes[1], ld, exps[1], lde, fb, 128)
        assert qe.qe_fp8_gemm_block(a, b, m, n, k, None, c[1], qe.F32, n) == "OK"
        torch.cuda.synchronize()
        by = torch.randint(-60, 61, (groups,), generator=g, device=d)
        exps[0][:, :groups] = (127 + by).to(torch.uint8)
        exps[1][:, :groups] = (127 - by).to(torch.uint8)
        assert qe.qe_fp8_gemm_block(a, b, m, n, k, None, c[2], qe.F32, n) == "OK"
    finally:
        assert qe.qe_set_gemm_tile(qe.TILE_AUTO) == "OK"
    assert float(c[0].abs().max()) > 0 and bool(c[0].isfinite().all())
    assert torch.equal(c[0], c[1]) and torch.equal(c[1], c[2])
