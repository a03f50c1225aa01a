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

hipError_t launch_block_gemm(const BlockGemmParams &p, hipStream_t s) {
  if (p.m <= 0 || p.n <= 0) return hipSuccess;
  if (p.fmt_a == 0 && p.fmt_b == 0) return launch_rows<0, 0>(p, s);
  if (p.fmt_a == 1 && p.fmt_b == 0) return launch_rows<1, 0>(p, s);
  if (p.fmt_a == 0 && p.fmt_b == 1) return launch_rows<0, 1>(p, s);
  return launch_rows<1, 1>(p, s);
}

}  // namespace qe
