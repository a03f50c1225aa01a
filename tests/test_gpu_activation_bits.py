"""Which bits the products with an epilogue share: with the plain product, between shapes, between calls."""
import pytest

from tests.gpu_util import dev, torch
from tests.libqe import need_lib

pytestmark = pytest.mark.gpu


def operands(d, m, n, k, seed=5):
    g = torch.Generator(device=d)
    g.manual_seed(seed)
    ld = (k + 15) // 16 * 16

    def codes(rows, sigma):
        q = torch.zeros((rows, ld), dtype=torch.uint8, device=d)
        q[:, :k] = (torch.randn((rows, k), generator=g, device=d) * sigma).to(torch.float8_e4m3fn).view(torch.uint8)
        return q
    return codes(m, 60.0), codes(n, 60.0), torch.tensor([1 / 64, 1 / 1024], device=d), ld


def plain(qe, a, b, s, ld, m, n, k, d):
    c = torch.zeros((m, n), device=d)
    assert qe.qe_fp8_gemm_tn(a, 0, ld, b, 0, ld, m, n, k, s[0:1], s[1:2], c, qe.F32, n, qe.INIT) == "OK"
    return c


def act(qe, a, b, s, ld, m, n, k, d):
    c = torch.zeros((m, n), device=d)
    assert qe.qe_fp8_gemm_act(a, 0, ld, b, 0, ld, m, n, k, s[0:1], s[1:2], None, c, qe.F32, n) == "OK"
    return c


@pytest.mark.parametrize("tile", ["TILE_AUTO", "TILE_256x256", "TILE_192x256"])
@pytest.mark.parametrize("m,n,k", [(300, 520, 384), (129, 700, 1000), (513, 4096, 2048), (64, 8192, 1500)])
def test_the_sums_are_the_plain_product_s(m, n, k, tile):
    qe, d = need_lib(), dev()
    a, b, s, ld = operands(d, m, n, k)
    want = plain(qe, a, b, s, ld, m, n, k, d)
    assert qe.qe_set_gemm_tile(getattr(qe, tile)) == "OK"
    try:
        got = act(qe, a, b, s, ld, m, n, k, d)
        torch.cuda.synchronize()
    finally:
        assert qe.qe_set_gemm_tile(qe.TILE_AUTO) == "OK"
    assert torch.equal(got, want)


@pytest.mark.parametrize("m,n,k", [(1, 4096, 4096), (16, 500, 2730), (50, 256, 6534), (200, 512, 12300)])
def test_a_split_reduction_repeats_its_bits(m, n, k):
    """And is as near to the exact sums as the plain product: both take the instruction's sums of 128 products, off by at
    most 1e-4 of the sum of their magnitudes (the plain GEMM's tests allow 1e-3 of the largest output)."""
    qe, d = need_lib(), dev()
    a, b, s, ld = operands(d, m, n, k)
    got = act(qe, a, b, s, ld, m, n, k, d)
    for _ in range(3):
        assert torch.equal(act(qe, a, b, s, ld, m, n, k, d), got)
    av, bv = (q[:, :k].contiguous().view(torch.float8_e4m3fn).double() for q in (a, b))
    exact = (av @ bv.t()) * float(s[0]) * float(s[1])
    size = (av.abs() @ bv.abs().t()) * float(s[0]) * float(s[1])
    assert bool(((got.double() - exact).abs() <= 1e-4 * size).all())
    assert bool(((plain(qe, a, b, s, ld, m, n, k, d).double() - exact).abs() <= 1e-4 * size).all())
