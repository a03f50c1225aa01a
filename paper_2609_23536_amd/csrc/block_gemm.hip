// FP8 products of operands with a scale for each block of 128 (gfx950):
//     Z = sum over K tiles b of 2^(ea[i][b] + eb[j][b]) sum_{r in b} A[i][r] B[j][r] + bias,
//     D = act(Z) + residual
// The kernels are those of the products with one scale per operand (act_tiles.h);
// the matrix instruction applies the scales, powers of two, to its products by
// itself (LdsScales in gemm_loops.h), so nothing is added to the sums' arithmetic.  A
// row's bytes are a 128th of its codes: from LDS, a word for four K tiles, they cost the
// large tiles 4%, the small ones, which read single bytes, up to 11% of their time.
// Bound by the matrix instructions from K = 4096 on (MI355X: 8192 x 8192 x 28672 1310 us,
// 2.9 PFLOP/s; 4096 x 4096 x 28672 325 us, one round of tiles), by each round's prologue
// and stores below (6144 x 4096 x 2048 with a residual 59 us, 1.75 PFLOP/s), for a few
// rows by the other operand's bytes (1 x 4096 x 14336 12.9 us, 4.6 TB/s).
#include "block_gemm.h"
#include "gemm_util.h"

namespace qe {
namespace {

constexpr int64_t kFewRows = 16;

// As for one scale per operand (few_blocks in act_gemm.hip); a launch holds less than
// 2^32 lanes, 512 of them a block.
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
  // The plain GEMM's cost model.
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
