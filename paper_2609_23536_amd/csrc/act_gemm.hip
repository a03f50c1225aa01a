// FP8 products whose epilogue goes on past the sum (gfx950):
//     plain:  Z = s A B^T + bias,  D = act(Z) + residual
//     gated:  G = sg A Bg^T,  U = su A Bu^T,  D = act(G) * U
// (s, sg, su: the products of the operands' scale inverses, sum_scale)
// and, for a backward pass, Z (or G and U) saved beside D in BF16 or 8 bits
// (act.h).  Everything after the sums stays in registers and FP32; D is rounded
// once.
//
// The K loops are those of the plain GEMM (gemm_loops.h).  A gated tile of BN
// operand rows holds BN/2 rows of either projection, in alternating blocks of
// 16: an MFMA block column of gates is followed by the block column of the same
// outputs' ups, in the same wave, so one pass over A serves both projections
// and act(G) * U needs nothing from another wave.  Loads: 16-row blocks alternate
// with bit 4 of the LDS row, which for every load of a wave is bit 1 of the wave, so
// a wave loads from one projection only, whose base is a scalar.
//
// Operands are addressed from the tile's own first row, so that neither they
// nor the outputs have a size limit past a tile's: a row stride below 2^23
// bytes (256 rows of it are 2^31).
//
// Epilogue.  Large tiles finish in the accumulators' own layout, one wave's block
// of rows at a time (see act_large_kernel).  Small tiles' accumulators go through
// LDS, 64 rows of the workgroup at a time, and come back row by row, four
// columns a lane, the eight lanes of a 32-column group sharing its maximum by
// lane permutes.
//
// MI355X: 8192 x 8192 x 28672 with a BF16 residual 1290-1340 us (2.9 PFLOP/s, as the
// plain product), gated 4096 x 14336 x 4096 with both projections saved in 8 bits
// 400-446 us, where the plain product of 28672 columns takes 379.  Bound by the MFMAs
// and, over short K, by the epilogue's bursts of output.
#include "act_tiles.h"

namespace qe {
namespace {

template <bool GATED, int FA, int FB, int BM, int BN>
__global__ __launch_bounds__(256) void act_large_kernel(ActGemmParams g, int tiles_m, int tiles_n) {
  act_large_tile<GATED, FA, FB, BM, BN>(g, tiles_m, tiles_n);
}

template <bool GATED, int FA, int FB, int BM, int BN, int S>
__global__ __launch_bounds__(256, (BM + BN) * BK * S > 81920 ? 1 : 2) void act_ring_kernel(ActGemmParams g, int tiles_m,
                                                                                           int tiles_n) {
  act_ring_tile<GATED, FA, FB, BM, BN, S>(g, tiles_m, tiles_n);
}

template <bool GATED, int FA, int FB, int OB, int W>
__global__ __launch_bounds__(64 * W) void act_rows_kernel(ActGemmParams g, int blocks_n) {
  act_rows_tile<GATED, FA, FB, OB, W>(g, blocks_n);
}

constexpr int64_t kFewRows = 16;
constexpr int kFewRowsTile = 0;  // in place of a GemmTile

// More rows, in blocks of 16, where the whole product has few blocks and a long
// reduction: a tile kernel then runs a handful of workgroups, each through all of
// K.  MI355X, us with the small tiles / so, every call on other weights (1 GB of
// them in turn, as a program of many layers has): 17 x 512 x 2048 8.1 / 8.1, x 4096
// 11.9 / 8.1, x 14336 30.6 / 17.2; 200 x 256 x 6534 18.0 / 8.5; 32 x 2048 x 20480 45 / 22;
// gated 112 x 128 x 8192 19.7 / 13.9; saved in 8 bits 200 x 256 x 14336 30.0 / 24.3.
// Past one workgroup per unit every block's operands come from the caches once
// more, and only long reductions win: 32 x 4096 x 13000 40.1 / 27.4, x 14336 33.5 /
// 32.6, x 28672 62.9 / 54.9; 369 x 256 x 4096 9.5 / 10.2, x 12300 42.5 / 19.7.
// (The same weights again and again, out of the caches: level up to K = 2048 and
// 1.03 to 2 times faster so beyond, but strides of whole lines lose past one
// workgroup per unit, 32 x 4096 x 14336 22.3 / 30.6, and gated or 8-bit saved, 17 x 512 x
// 14336 18.2 / 23.3.)  Gated products saved in 8 bits take 32 outputs a workgroup
// and lose: 50 x 64 x 6534 11.5 / 15.2.
bool few_blocks(const ActGemmParams &p) {
  if (p.m <= kFewRows) return true;
  const bool gated = p.b2 != nullptr, wide = p.z.kind == kSavedI8;
  const int64_t blocks = (p.m + 15) / 16 * ((p.n + (wide ? 31 : 15)) / (wide ? 32 : 16));
  if (p.k <= 1024 || (gated && wide)) return false;
  const int64_t cus = compute_units();
  return blocks <= cus || (blocks <= 2 * cus && p.k > 12288 && !gated && !wide);
}

// One workgroup for 16 outputs (32 where they are saved in 8 bits, whose groups
// have 32 columns).  Eight waves keep the most bytes in flight, but up to 16 K
// tiles four waves have them all in flight in one go and start sooner.  MI355X,
// one row, us with 4 / 8 waves: 7936 x 739 (6 K tiles, 7 rows) 4.8 / 5.7, gated
// 2730 x 1365 (11) 4.1 / 5.2, 4096 x 4096 (32) 7.7 / 6.0, gated 14336 x 4096 28.5 /
// 24.9, 8192 x 28672 45.1 / 41.9.
// Against the small tiles, MI355X, us small tile / so, other weights every call:
// one row 512 x 14336 30.1 / 12.8, 8192 x 4096 13.4 / 9.9, 14336 x 8192 27.7 / 24.5, gated
// 14336 x 4096 28.5 / 25.0, gated 14336 x 8192 46.4 / 44.7, but 14336 x 14336 39.3 / 42.7;
// sixteen 512 x 14336 30.5 / 17.1, gated 14336 x 4096 28.1 / 27.8, but 14336 x 8192 28.0 /
// 33.8.  Two row blocks a wave for 32 rows: 21.8 -> 23.6 and gated 30.8 -> 38.0, so not there.
template <bool GATED, int FA, int FB>
hipError_t launch_few_rows(const ActGemmParams &p, hipStream_t s) {
  const bool wide = p.z.kind == kSavedI8, few = p.k <= 16 * BK;
  const int blocks_n = int((p.n + (wide ? 31 : 15)) / (wide ? 32 : 16));
  const dim3 grid(unsigned((p.m + 15) / 16) * unsigned(blocks_n));
  if (wide)
    return few ? klaunch(act_rows_kernel<GATED, FA, FB, 2, 4>, grid, dim3(256), 0, s, p, blocks_n)
               : klaunch(act_rows_kernel<GATED, FA, FB, 2, 8>, grid, dim3(512), 0, s, p, blocks_n);
  return few ? klaunch(act_rows_kernel<GATED, FA, FB, 1, 4>, grid, dim3(256), 0, s, p, blocks_n)
             : klaunch(act_rows_kernel<GATED, FA, FB, 1, 8>, grid, dim3(512), 0, s, p, blocks_n);
}

template <bool GATED, int FA, int FB>
hipError_t launch_tile(int tile, const ActGemmParams &p, hipStream_t s) {
  if (tile == kFewRowsTile) return launch_few_rows<GATED, FA, FB>(p, s);
  const dim3 block(256);
  int tm = 0, tn = 0;
  auto grid = [&](int bm, int bn) {
    tm = int((p.m + bm - 1) / bm);
    tn = int((p.n + (GATED ? bn / 2 : bn) - 1) / (GATED ? bn / 2 : bn));
    return dim3(unsigned(tm) * unsigned(tn));
  };
#define QE_RING(BM, BN, S) \
  { const dim3 n = grid(BM, BN); return klaunch(act_ring_kernel<GATED, FA, FB, BM, BN, S>, n, block, 0, s, p, tm, tn); }
#define QE_LARGE(BM, BN) \
  { const dim3 n = grid(BM, BN); return klaunch(act_large_kernel<GATED, FA, FB, BM, BN>, n, block, 0, s, p, tm, tn); }
  switch (tile) {
    case kTile64x64: QE_RING(64, 64, 4)
    case kTile128x64: QE_RING(128, 64, 3)
    case kTile128x64Deep: QE_RING(128, 64, 6)
    case kTile64x128: QE_RING(64, 128, 3)
    case kTile64x128Deep: QE_RING(64, 128, 6)
    case kTile128x128: QE_RING(128, 128, 2)
    case kTile128x128Deep: QE_RING(128, 128, 4)
    case kTile192x256: QE_LARGE(192, 256)
    default: QE_LARGE(256, 256)
  }
#undef QE_RING
#undef QE_LARGE
}

template <bool GATED>
hipError_t launch_fmts(int tile, const ActGemmParams &p, hipStream_t s) {
  if (p.fmt_a == 0 && p.fmt_b == 0) return launch_tile<GATED, 0, 0>(tile, p, s);
  if (p.fmt_a == 1 && p.fmt_b == 0) return launch_tile<GATED, 1, 0>(tile, p, s);
  if (p.fmt_a == 0 && p.fmt_b == 1) return launch_tile<GATED, 0, 1>(tile, p, s);
  return launch_tile<GATED, 1, 1>(tile, p, s);
}

}  // namespace

hipError_t launch_act_gemm(const ActGemmParams &p, hipStream_t s) {
  if (p.m <= 0 || p.n <= 0) return hipSuccess;
  const bool gated = p.b2 != nullptr;
  // The plain GEMM's cost model, on a product of as many operand rows.
  GemmParams g;
  memset(&g, 0, sizeof(g));
  g.m = p.m;
  g.n = gated ? 2 * p.n : p.n;
  g.k = p.k;
  g.c = p.c;
  g.ldc = p.ldc;
  g.out = p.c_bf16 ? 1 : 0;
  constexpr unsigned kShapes = 1u << kTile256x256 | 1u << kTile192x256 | 1u << kTile64x64 | 1u << kTile128x64 |
                               1u << kTile128x64Deep | 1u << kTile64x128 | 1u << kTile64x128Deep | 1u << kTile128x128 |
                               1u << kTile128x128Deep;
  const int force = gemm_tile_override();
  if (force == kTileAuto && few_blocks(p))
    return gated ? launch_fmts<true>(kFewRowsTile, p, s) : launch_fmts<false>(kFewRowsTile, p, s);
  const int tile = force == kTileAuto ? choose_gemm_tile(g, kShapes) : (force == kTile192x256 ? kTile192x256 : kTile256x256);
  return gated ? launch_fmts<true>(tile, p, s) : launch_fmts<false>(tile, p, s);
}

}  // namespace qe
