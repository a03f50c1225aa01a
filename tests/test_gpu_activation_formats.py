"""Products with an epilogue in every pair of FP8 formats, on each kind of small tile and of few-rows kernel."""
import pytest

from tests.act_tiles import TILES
from tests.gpu_util import dev
from tests.libqe import need_lib
from tests.test_gpu_activation import check_gated, check_product

pytestmark = pytest.mark.gpu
FORMATS = [(1, 0), (0, 1), (1, 1)]


@pytest.mark.parametrize("fa,fb", FORMATS)
@pytest.mark.parametrize("tile", TILES, ids=lambda t: t[0][4:])
def test_every_small_tile(tile, fa, fb):
    _, gated, m, n, k = tile
    if gated:
        check_gated(need_lib(), dev(), (m, n, k), 7, "silu", "bf16", "none", fa, fb)
    else:
        check_product(need_lib(), dev(), (m, n, k), 7, "silu", "f32", "bf16", "bf16", "none", fa, fb)


@pytest.mark.parametrize("fa,fb", FORMATS)
@pytest.mark.parametrize("saved", ["none", "i8"])
@pytest.mark.parametrize("shape", [(1, 100, 300), (16, 70, 4100), (50, 70, 2100)], ids=str)
def test_few_rows(shape, saved, fa, fb):
    """Four and eight waves, with 16 and (saved in 8 bits) 32 outputs a workgroup."""
    check_product(need_lib(), dev(), shape, 8, "none", "bf16", "f32", "f32", saved, fa, fb, 1)
    check_gated(need_lib(), dev(), shape, 9, "silu", "bf16", saved, fa, fb, 3)
