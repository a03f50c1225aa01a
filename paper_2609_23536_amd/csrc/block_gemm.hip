// FP8 products of operands with a scale for each block of 128 (gfx950):
//     Z = sum over K tiles b of 2^(ea[i][b] + eb[j][b]) sum_{r in b} A[i][r] B[j][r] + bias,
//     D = act(Z) + residual
// The kernels are those of the products with one scale per operand (act_tiles.h);
// the matrix instruction applies the scales, powers of two, to its products by
// itself (LdsScales in gemm_loops.h), so nothing is added to the sums' arithmetic.
#include "act_tiles.h"

namespace qe {
namespace {

template <int FA, int FB, int OB, int W>
__global__ __launch_bounds__(64 * W) void block_rows_kernel(BlockGemmParams g, int blocks_n) {
  act_rows_tile<false, FA, FB, OB, W>(g, blocks_n);
}

template <int FA, int FB, int BM, int BN>
__global__ __launch_bounds__(256) void block_large_kernel(BlockGemmParams g, int tiles_m, int tiles_n) {
  act_large_tile<false, FA, FB, BM, BN>(g, tiles_m, tiles_n);
}

template <int FA, int FB, int BM, int BN, int S>
__global__ __launch_bounds__(256, (BM + BN) * BK * S > 81920 ? 1 : 2) void block_ring_kernel(BlockGemmParams g, int tiles_m,
                                                                                             int tiles_n) {
  act_ring_tile<false, FA, FB, BM, BN, S>(g, tiles_m, tiles_n);
}

constexpr int64_t kFewRows = 16;
constexpr int kFewRowsTile = 0;  // in place of a GemmTile

// As for one scale per operand (few_blocks in act_gemm.hip); a launch holds less than
// 2^32 lanes, 512 of them a block.
bool few_blocks(const BlockGemmParams &p) {
  const bool wide = p.z.kind == kSavedI8;
  const int64_t blocks = (p.m + 15) / 16 * ((p.n + (wide ? 31 : 15)) / (wide ? 32 : 16)), cus = compute_units();
  if (p.m <= kFewRows) return blocks < int64_t(1) << 23;
  if (p.k <= 1024) return false;
  return blocks <= cus || (blocks <= 2 * cus && p.k > 12288 && !wide);
}

template <int FA, int FB>
hipError_t launch_rows(const BlockGemmParams &p, hipStream_t s) {
  const bool wide = p.z.kind == kSavedI8, few = p.k <= 16 * BK;
  const int blocks_n = int((p.n + (wide ? 31 : 15)) / (wide ? 32 : 16));
  const dim3 grid(unsigned((p.m + 15) / 16) * unsigned(blocks_n));
  if (wide)
    return few ? klaunch(block_rows_kernel<FA, FB, 2, 4>, grid, dim3(256), 0, s, p, blocks_n)
               : klaunch(block_rows_kernel<FA, FB, 2, 8>, grid, dim3(512), 0, s, p, blocks_n);
  return few ? klaunch(block_rows_kernel<FA, FB, 1, 4>, grid, dim3(256), 0, s, p, blocks_n)
             : klaunch(block_rows_kernel<FA, FB, 1, 8>, grid, dim3(512), 0, s, p, blocks_n);
}

template <int FA, int FB>
hipError_t launch_tile(int tile, const BlockGemmParams &p, hipStream_t s) {
  if (tile == kFewRowsTile) return launch_rows<FA, FB>(p, s);
  const dim3 block(256);
  auto tiles = [&](auto *kernel, int bm, int bn) {
    const int tm = int((p.m + bm - 1) / bm), tn = int((p.n + bn - 1) / bn);
    return klaunch(kernel, dim3(unsigned(tm) * unsigned(tn)), block, 0, s, p, tm, tn);
  };
  switch (tile) {
    case kTile64x64: return tiles(block_ring_kernel<FA, FB, 64, 64, 4>, 64, 64);
    case kTile128x64: return tiles(block_ring_kernel<FA, FB, 128, 64, 3>, 128, 64);
    case kTile128x64Deep: return tiles(block_ring_kernel<FA, FB, 128, 64, 6>, 128, 64);
    case kTile64x128: return tiles(block_ring_kernel<FA, FB, 64, 128, 3>, 64, 128);
    case kTile64x128Deep: return tiles(block_ring_kernel<FA, FB, 64, 128, 6>, 64, 128);
    case kTile128x128: return tiles(block_ring_kernel<FA, FB, 128, 128, 2>, 128, 128);
    case kTile128x128Deep: return tiles(block_ring_kernel<FA, FB, 128, 128, 4>, 128, 128);
    case kTile192x256: return tiles(block_large_kernel<FA, FB, 192, 256>, 192, 256);
    default: return tiles(block_large_kernel<FA, FB, 256, 256>, 256, 256);
  }
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
  if (p.fmt_a == 0 && p.fmt_b == 0) return launch_tile<0, 0>(tile, p, s);
  if (p.fmt_a == 1 && p.fmt_b == 0) return launch_tile<1, 0>(tile, p, s);
  if (p.fmt_a == 0 && p.fmt_b == 1) return launch_tile<0, 1>(tile, p, s);
  return launch_tile<1, 1>(tile, p, s);
}

}  // namespace qe
