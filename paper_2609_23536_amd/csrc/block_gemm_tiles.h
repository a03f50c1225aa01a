// Kernels of the FP8 products with a scale for each block of 128 (block_gemm.hip), for one
// pair of operand formats a source file.
#pragma once

#include "act_tiles.h"
#include "block_gemm.h"

namespace qe {
namespace {

template <int FA, int FB, int OB, int W>
__global__ __launch_bounds__(64 * W) void block_rows_kernel(BlockGemmParams g, int blocks_n) {
  act_rows_tile<false, FA, FB, OB, W>(g, blocks_n);
}

template <int FA, int FB, int BM, int BN, TileOut OUT>
__global__ __launch_bounds__(256) void block_large_kernel(BlockGemmParams g, int tiles_m, int tiles_n) {
  act_large_tile<false, FA, FB, BM, BN, OUT>(g, tiles_m, tiles_n);
}

template <int FA, int FB, int BM, int BN, int S>
__global__ __launch_bounds__(256, (BM + BN) * BK * S > 81920 ? 1 : 2) void block_ring_kernel(BlockGemmParams g, int tiles_m,
                                                                                             int tiles_n) {
  act_ring_tile<false, FA, FB, BM, BN, S>(g, tiles_m, tiles_n);
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

}  // namespace

template <int FA, int FB>
hipError_t launch_block_tile(int tile, const BlockGemmParams &p, hipStream_t s) {
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
    case kTile192x256: return tiles(p.c_bf16 ? block_large_kernel<FA, FB, 192, 256, kBF16> : block_large_kernel<FA, FB, 192, 256, kF32>, 192, 256);
    default: return tiles(p.c_bf16 ? block_large_kernel<FA, FB, 256, 256, kBF16> : block_large_kernel<FA, FB, 256, 256, kF32>, 256, 256);
  }
}

}  // namespace qe
