// FP8 products of operands with a scale for each block of 128 (gfx950):
//     Z = sum over K tiles b of 2^(ea[i][b] + eb[j][b]) sum_{r in b} A[i][r] B[j][r] + bias,
//     D = act(Z) + residual
// The kernels are those of the products with one scale per operand (act_tiles.h);
// the matrix instruction applies the scales, powers of two, to its products by
// itself (LdsScales in gemm_loops.h), so nothing is added to the sums' arithmetic: on one
// tile they have the bits of the product with one scale.  That arithmetic is the
// instruction's, which aligns the 128 products of a step to their largest one: its sums are
// 1.5e-5 of their size off on random data and 3.4e-5 where one channel in a thousand is
// twenty times larger (FP32 products 1e-7).  That is the price of FP8 at its full rate, and
// far below half a step of a BF16 output, 2^-9 of its size or more.
// A row's bytes are a 128th of its codes: from LDS, a word for four K tiles, they cost the
// large tiles 4%, the small ones, which read single bytes, up to 11% of their time.
// Bound by the matrix instructions from K = 4096 on (MI355X: 8192 x 8192 x 28672 1268-1314
// us, 3.0 PFLOP/s; 4096 x 4096 x 28672 316-326 us, one round of tiles), by each round's
// prologue and stores below (6144 x 4096 x 2048 accumulated in place 52 us, 2.0 PFLOP/s), for
// a few rows by the other operand's bytes (1 x 4096 x 14336 12.9 us, 4.6 TB/s).
#include "block_gemm.h"
#include "gemm_util.h"

namespace qe {
namespace {

constexpr int64_t kFewRows = 16;

// The rule of the products with one scale (few_blocks in act_gemm.hip), as it was fitted
// there; a launch holds less than 2^32 lanes, 512 of them a block.  With block scales on
// cold weights, MI355X, us tile / so: one row 512 x 14336 31.6 / 12.4, 4096 x 14336 32.1 /
// 14.3, 14336 x 8192 27.3 / 26.2, 8192 x 28672 68.6 / 50.5; sixteen 4096 x 14336 32.6 / 18.2,
// but 14336 x 8192 27.8 / 35.9; 17 x 512 x 2048 8.4 / 5.2, 200 x 256 x 6534 27.8 / 10.0, 32 x
// 2048 x 20480 47.5 / 24.4, 32 x 4096 x 28672 65.0 / 60.6, 369 x 256 x 12300 49.5 / 25.2; not
// so by this rule though faster: 200 x 256 x 1024 5.7 / 4.0, 17 x 512 x 1000 6.2 / 5.0, 369 x
// 256 x 4096 12.9 / 11.1; 48 x 4096 x 14336 36.5 / 42.9.
bool few_blocks(const BlockGemmParams &p) {
  const bool wide = p.z.kind == kSavedI8;
  const int64_t blocks = (p.m + 15) / 16 * ((p.n + (wide ? 31 : 15)) / (wide ? 32 : 16)), cus = compute_units();
  if (p.m <= kFewRows) return blocks < int64_t(1) << 23;
  if (p.k <= 1024) return false;
  return blocks <= cus || (blocks <= 2 * cus && p.k > 12288 && !wide);
}

}  // namespace

hipError_t launch_block_gemm(const BlockGemmParams &p, hipStream_t s) {
  if (p.m <= 0 || p.n <= 0) return hipSuccess;
  // The plain GEMM's cost model, fitted without scales.  Over 90 products (M 200 .. 4000, N 256 ..
  // 4096, K 256 .. 4000, MI355X, cold operands) its choice takes 1.03 times the fastest tile's
  // time in the geometric mean; at worst 1.27 (4000 x 1000 x 256: 11.8, 128 x 64 9.3).
  GemmParams g;
  memset(&g, 0, sizeof(g));
  g.m = p.m;
  g.n = p.n;
  g.k = p.k;
  g.c = p.c;
  g.ldc = p.ldc;
  g.out = p.c_bf16 ? 1 : 0;
  constexpr unsigned kShapes = 1u << kTile256x256 | 1u << kTile192x256 | 1u << kTile64x64 | 1u << kTile128x64 |
                               1u << kTile128x64Deep | 1u << kTile64x128 | 1u << kTile64x128Deep | 1u << kTile128x128 |
                               1u << kTile128x128Deep;
  const int force = gemm_tile_override();
  const int tile = force == kTileAuto ? (few_blocks(p) ? kFewRowsTile : choose_gemm_tile(g, kShapes))
                                      : (force == kTile192x256 ? kTile192x256 : kTile256x256);
  if (p.fmt_a == 0 && p.fmt_b == 0) return launch_block_tile<0, 0>(tile, p, s);
  if (p.fmt_a == 1 && p.fmt_b == 0) return launch_block_tile<1, 0>(tile, p, s);
  if (p.fmt_a == 0 && p.fmt_b == 1) return launch_block_tile<0, 1>(tile, p, s);
  return launch_block_tile<1, 1>(tile, p, s);
}

}  // namespace qe
