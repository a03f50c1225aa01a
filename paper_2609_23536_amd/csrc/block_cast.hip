// FP8 cast with a power-of-two scale for each block of 128 values (gfx950),
// row-wise (blocks along a row) and transposed (blocks along a column) in one
// pass, or with one scale per 128 x 128 block for both orders.
//
// One workgroup of 256 lanes per 128 x 128 tile, which holds whole blocks of either
// kind: a lane keeps its 64 values in registers, so the maxima come first and the
// codes after them without a second read.  A lane holds eight neighbouring values of
// rows tid / 16 + 16 s, s = 0 .. 7: a row's block is 16 neighbouring lanes (four lane
// exchanges), a column's is eight values of a lane, four lanes of a wave and the four
// waves (two lane exchanges and 2 KB of LDS).  The transposed codes go through LDS as
// in quantize.hip.  The values may be a norm's output, computed on the fly from its
// input and the rows' factors.
#include "block_scale.h"

namespace qe {
namespace {

constexpr int kSteps = 8, kRowStep = 16;  // a lane's rows: tid / 16 + 16 s

template <bool BF16, int FMT, bool SQUARE, bool NORM>
__global__ __launch_bounds__(kThreads) void block_cast_kernel(BlockCastParams p, int tiles_c) {
  __shared__ __attribute__((aligned(16))) uint8_t tile[kTile * kTile];
  __shared__ __attribute__((aligned(16))) float part[4][kTile];
  const int tid = threadIdx.x, wave = tid >> 6, lr = tid >> 4, cl = (tid & 15) * 8;
  const int tr = int(blockIdx.x) / tiles_c, tc = int(blockIdx.x) % tiles_c;
  const int64_t r0 = int64_t(tr) * kTile, c0 = int64_t(tc) * kTile;
  const int rows = int(min(int64_t(kTile), p.rows - r0)), cols = int(min(int64_t(kTile), p.cols - c0));
  const int n = max(0, min(8, cols - cl));  // the lane's columns that exist
  float v[kSteps][8];
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const int row = lr + kRowStep * s;
    load8(row_of(p.in, BF16, r0 + row), BF16, uint32_t(c0) + cl, row < rows ? n : 0, v[s]);
  }
  if constexpr (NORM) {
    float w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = 1.0f;
    if (p.weight != nullptr) {
      load8(p.weight, p.weight_bf16 != 0, uint32_t(c0) + cl, n, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] += p.offset;
    }
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int row = lr + kRowStep * s;
      const float f = row < rows ? p.rstd[r0 + row] : 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[s][e] = e < n ? v[s][e] * f * w[e] : 0.0f;
    }
  }
  // maxima
  float row_max[kSteps], col_max[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) col_max[e] = 0.0f;
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    row_max[s] = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float a = __builtin_fabsf(v[s][e]);
      row_max[s] = nan_max(row_max[s], a);
      if constexpr (!SQUARE) col_max[e] = nan_max(col_max[e], a);
    }
  }
  const bool transposed = p.col.data != nullptr;
  float all = 0.0f;
  if constexpr (SQUARE) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) all = nan_max(all, row_max[s]);
    all = max_lanes_by16(max_lanes16(all));
    if ((tid & 63) == 0) part[0][wave] = all;
    __syncthreads();
    all = nan_max(nan_max(part[0][0], part[0][1]), nan_max(part[0][2], part[0][3]));
  } else {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) row_max[s] = max_lanes16(row_max[s]);
    if (transposed) {
#pragma unroll
      for (int e = 0; e < 8; ++e) col_max[e] = max_lanes_by16(col_max[e]);
      if ((tid & 63) < 16) {
#pragma unroll
        for (int e = 0; e < 8; ++e) part[wave][cl + e] = col_max[e];
      }
      __syncthreads();
    }
  }
  const uint32_t all_byte = block_byte<FMT>(all);
  // row-wise codes; of square blocks the transposed ones are the same
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const int row = lr + kRowStep * s;
    const uint32_t byte = SQUARE ? all_byte : block_byte<FMT>(row_max[s]);
    const float mult = block_mult(byte);
    const uint32_t lo = block_codes<FMT>(v[s], mult), hi = block_codes<FMT>(v[s] + 4, mult);
    if constexpr (SQUARE)
      *reinterpret_cast<uint2 *>(tile + lds_chunk_offset<16>(row, cl >> 4) + (cl & 15)) = make_uint2(lo, hi);
    if (p.row.data != nullptr && row < rows) {
      store_codes8(p.row.data + (r0 + row) * p.row.ld + c0 + cl, n, lo, hi);
      if (!SQUARE && cl == 0) p.row.exps[(r0 + row) * p.row.ld_exps + tc] = uint8_t(byte);
    }
  }
  if (SQUARE && tid == 0) {
    if (p.row.data != nullptr) p.row.exps[tr * p.row.ld_exps + tc] = uint8_t(all_byte);
    if (transposed) p.col.exps[tc * p.col.ld_exps + tr] = uint8_t(all_byte);
  }
  if (!transposed) return;
  if constexpr (!SQUARE) {
    float mult[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float m = nan_max(nan_max(part[0][cl + e], part[1][cl + e]), nan_max(part[2][cl + e], part[3][cl + e]));
      const uint32_t byte = block_byte<FMT>(m);
      mult[e] = block_mult(byte);
      if (lr == 0 && e < n) p.col.exps[(c0 + cl + e) * p.col.ld_exps + tr] = uint8_t(byte);
    }
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int row = lr + kRowStep * s;
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = v[s][e] * mult[e];
      *reinterpret_cast<uint2 *>(tile + lds_chunk_offset<16>(row, cl >> 4) + (cl & 15)) =
          make_uint2(enc4_in_range<FMT>(x[0], x[1], x[2], x[3]), enc4_in_range<FMT>(x[4], x[5], x[6], x[7]));
    }
  }
  __syncthreads();
  // Lane (rb, cq): rows 16 rb .. + 15 of columns 4 cq .. + 3, as in quantize.hip.
  const int rb = tid & 7, cq = tid >> 3;
  uint32_t d[16];
#pragma unroll
  for (int i = 0; i < 16; ++i)
    d[i] = *reinterpret_cast<const uint32_t *>(tile + lds_chunk_offset<16>(rb * 16 + i, cq >> 2) + ((cq & 3) << 2));
  const int left = rows - rb * 16;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint32_t w[4];
#pragma unroll
    for (int q = 0; q < 4; ++q)
      w[q] = byte_of(d[4 * q], j) | (byte_of(d[4 * q + 1], j) << 8) | (byte_of(d[4 * q + 2], j) << 16) |
             (byte_of(d[4 * q + 3], j) << 24);
    if (4 * cq + j >= cols) continue;
    uint8_t *dst = p.col.data + (c0 + 4 * cq + j) * p.col.ld + r0 + rb * 16;
    if (left >= 16) {
      *reinterpret_cast<u32x4_out *>(dst) = u32x4_out{w[0], w[1], w[2], w[3]};
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (e < left) dst[e] = uint8_t(byte_of(w[e / 4], e % 4));
    }
  }
}

template <bool BF16, int FMT>
hipError_t launch_fmt(const BlockCastParams &p, hipStream_t s) {
  const int64_t tiles_r = (p.rows + kTile - 1) / kTile, tiles_c = (p.cols + kTile - 1) / kTile;
  const dim3 grid{unsigned(tiles_r * tiles_c)}, block(kThreads);
  const bool square = (p.row.data != nullptr ? p.row : p.col).row_shift != 0;
  if (p.rstd != nullptr) return klaunch(block_cast_kernel<BF16, FMT, false, true>, grid, block, 0, s, p, int(tiles_c));
  return square ? klaunch(block_cast_kernel<BF16, FMT, true, false>, grid, block, 0, s, p, int(tiles_c))
                : klaunch(block_cast_kernel<BF16, FMT, false, false>, grid, block, 0, s, p, int(tiles_c));
}

}  // namespace

hipError_t launch_block_cast(const BlockCastParams &p, hipStream_t s) {
  if (p.rows <= 0 || p.cols <= 0 || (p.row.data == nullptr && p.col.data == nullptr)) return hipSuccess;
  const int fmt = (p.row.data != nullptr ? p.row : p.col).fmt;
  if (p.in.bf16) return fmt == 0 ? launch_fmt<true, 0>(p, s) : launch_fmt<true, 1>(p, s);
  return fmt == 0 ? launch_fmt<false, 0>(p, s) : launch_fmt<false, 1>(p, s);
}

}  // namespace qe
