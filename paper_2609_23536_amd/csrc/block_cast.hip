// FP8 cast with a power-of-two scale for each block of 128 values (gfx950),
// row-wise (blocks along a row) and transposed (blocks along a column) in one
// pass, or with one scale per 128 x 128 block for both orders.
//
// One workgroup of 256 lanes per 128 x 128 tile, which holds whole blocks of either
// kind: a lane keeps its 64 values in registers, so the maxima come first and the
// codes after them without a second read.  A lane holds two quads of columns of eight
// neighbouring rows: a row's block is 16 neighbouring lanes, a column's is eight values
// of a lane, four lanes of a wave and the four waves.  The conversion instruction takes
// the scale itself and converts two values: two of a row, or, for the transposed codes,
// the same column's of two rows, so that a lane has eight neighbouring codes of each of
// its columns.  Those go through LDS, column by column, and leave as 128-byte runs.  The
// values may be a norm's output, computed on the fly from its input and the rows' factors
// (for the transposed codes alone: the row-wise ones left with the norm).
//
// Of BF16 values the maxima are taken on pairs of 16-bit patterns with the sign off,
// which order like the values (NaN above infinity), and no value is widened at all.
// Bound by memory: MI355X, both orders, BF16 4096 x 14336 51.5 us (4.6 TB/s), 57344 x 8192
// in square blocks 347 (5.4 TB/s).
#include "block_scale.h"
#include "gemm_util.h"

namespace qe {
namespace {

constexpr int kRows = 8;  // of a lane

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
template <int CTRL>
__device__ __forceinline__ uint32_t max_u16x2_dpp(uint32_t v) {
  return max_u16x2(v, uint32_t(__builtin_amdgcn_mov_dpp(int(v), CTRL, 0xf, 0xf, true)));
}
// block_byte of the upper half of a float
template <int FMT>
__device__ __forceinline__ uint32_t block_byte16(uint32_t a) {
  const int b = int((a + 0x1fu) >> 7) - (FMT == 0 ? 8 : 15);
  return a >= 0x7f80u ? 255u : uint32_t(b < 1 ? 1 : b);
}
// Eight bytes of transposed codes, rows 8 rg .. of column col, in LDS: 128 bytes a
// column, its 16-byte chunks turned by the column's eight and the upper 64 columns in
// the odd places, so that neither a wave's writes (16 lanes with every eighth column,
// four groups of rows) nor its reads (eight columns' chunks) meet in a bank twice.
__device__ __forceinline__ uint32_t turned(int col, int chunk) {
  return uint32_t(col ^ (col >> 6)) * kTile + uint32_t((chunk ^ (col >> 3)) & 7) * 16u;
}

// A lane's values.  BF16: as stored, two to a word; else as floats.
template <bool PACKED>
struct Values {
  uint32_t w[kRows][PACKED ? 4 : 8];
  __device__ __forceinline__ float f(int s, int e) const { return __uint_as_float(w[s][PACKED ? 0 : e]); }
};

// offset + weight of four columns, n of which exist (1 without weights).
__device__ __forceinline__ void load_weights4(const BlockCastParams &p, int64_t at, int n, float *f) {
#pragma unroll
  for (int e = 0; e < 4; ++e) f[e] = 1.0f;
  if (p.weight == nullptr) return;
  if (p.weight_bf16) {
    const uint16_t *w = static_cast<const uint16_t *>(p.weight) + at;
    if (n >= 4) {
      typedef unsigned int u32x2_in __attribute__((ext_vector_type(2), aligned(2)));
      const u32x2_in x = *reinterpret_cast<const u32x2_in *>(w);
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] = __uint_as_float(e % 2 == 0 ? x[e / 2] << 16 : x[e / 2] & 0xffff0000u);
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e) f[e] = e < n ? bf16_to_f32(w[e]) : 0.0f;
    }
  } else {
    const float *w = static_cast<const float *>(p.weight) + at;
    if (n >= 4) {
      const f32x4_in x = *reinterpret_cast<const f32x4_in *>(w);
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] = x[e];
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e) f[e] = e < n ? w[e] : 0.0f;
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) f[e] += p.offset;
}

// How a launch goes about its tiles.
enum CastHow { kByXcd = 1, kRowLines = 2, kColLines = 4 };

template <bool BF16, int FMT, bool SQUARE, bool NORM, bool EDGE>
__device__ __forceinline__ void cast_tile(const BlockCastParams &p, int tr, int tc, int how, uint8_t *tile, uint32_t *part) {
  constexpr bool PACKED = BF16 && !NORM;
  constexpr int HI = BF16 ? 4 : 64;  // from a lane's first quad of columns to its second
  const int tid = threadIdx.x, wave = tid >> 6, rg = tid >> 4, cl = (tid & 15) * (BF16 ? 8 : 4);
  const int64_t r0 = int64_t(tr) * kTile, c0 = int64_t(tc) * kTile;
  const int rows = EDGE ? int(min(int64_t(kTile), p.rows - r0)) : kTile, cols = EDGE ? int(min(int64_t(kTile), p.cols - c0)) : kTile;
  auto col_of = [&](int e) { return cl + (e < 4 ? e : HI + e - 4); };

  // Loads, all in flight together.  At the matrix's edge they may run into what lies
  // between two rows, masked below, but not past its last element.
  Values<PACKED> v;
  u32x4_in raw[kRows][BF16 ? 1 : 2];
  const int64_t end = (p.rows - 1) * p.in.ld + p.cols;
  constexpr int EPL = BF16 ? 8 : 4;
#pragma unroll
  for (int s = 0; s < kRows; ++s)
#pragma unroll
    for (int h = 0; h < (BF16 ? 1 : 2); ++h) {
      const int row = rg * kRows + s, c = cl + h * HI;
      const int64_t at = (r0 + row) * p.in.ld + c0 + c;
      const char *src = static_cast<const char *>(p.in.data) + at * (BF16 ? 2 : 4);
      if (!EDGE || (row < rows && c < cols && at + EPL <= end)) {
        raw[s][h] = *reinterpret_cast<const u32x4_in *>(src);
      } else {
        raw[s][h] = u32x4_in{0u, 0u, 0u, 0u};
        const int n = row < rows ? cols - c : 0;
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
          if (e >= n) break;
          if constexpr (BF16)
            raw[s][h][e / 2] |= uint32_t(reinterpret_cast<const uint16_t *>(src)[e]) << (16 * (e % 2));
          else
            raw[s][h][e] = reinterpret_cast<const uint32_t *>(src)[e];
        }
      }
    }
  float weight[NORM ? 8 : 1], rstd[NORM ? kRows : 1];
  if constexpr (NORM) {
#pragma unroll
    for (int h = 0; h < 2; ++h) load_weights4(p, c0 + cl + h * HI, EDGE ? cols - cl - h * HI : 4, weight + 4 * h);
#pragma unroll
    for (int s = 0; s < kRows; ++s) rstd[s] = !EDGE || rg * kRows + s < rows ? p.rstd[r0 + rg * kRows + s] : 0.0f;
  }
#pragma unroll
  for (int s = 0; s < kRows; ++s) {
    if constexpr (PACKED) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        v.w[s][q] = raw[s][0][q];
        if (EDGE) {
          const int left = cols - cl - 2 * q;  // columns of the pair that exist
          v.w[s][q] &= left >= 2 ? 0xffffffffu : (left == 1 ? 0xffffu : 0u);
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float x = BF16 ? __uint_as_float(e % 2 == 0 ? raw[s][0][e / 2] << 16 : raw[s][0][e / 2] & 0xffff0000u) : __uint_as_float(raw[s][BF16 ? 0 : e / 4][e % 4]);
        if constexpr (NORM) x = x * rstd[s] * weight[e];
        if (EDGE) x = col_of(e) < cols ? x : 0.0f;
        v.w[s][e] = __float_as_uint(x);
      }
    }
  }

  // The blocks' bytes: row_byte of the lane's rows, col_byte of its columns.
  const bool transposed = p.col.data != nullptr;
  uint32_t row_byte[kRows], col_byte[8];
  if constexpr (PACKED) {
    uint32_t row_max[kRows], col_max[4] = {0u, 0u, 0u, 0u};  // two rows (below), two columns a word
#pragma unroll
    for (int s = 0; s < kRows; ++s) {
      uint32_t a[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        a[q] = v.w[s][q] & 0x7fff7fffu;
        if (!SQUARE) col_max[q] = max_u16x2(col_max[q], a[q]);
      }
      row_max[s] = max_u16x2(max_u16x2(a[0], a[1]), max_u16x2(a[2], a[3]));
    }
#pragma unroll
    for (int s = 0; s < kRows; s += 2) {  // the halves of a row's word meet: row s low, row s + 1 high
      const uint32_t lo = __builtin_amdgcn_perm(row_max[s + 1], row_max[s], 0x05040100u);
      const uint32_t hi = __builtin_amdgcn_perm(row_max[s + 1], row_max[s], 0x07060302u);
      uint32_t m = max_u16x2(lo, hi);
      if constexpr (!SQUARE) {
        m = max_u16x2_dpp<0x140>(max_u16x2_dpp<0x141>(max_u16x2_dpp<0x4e>(max_u16x2_dpp<0xb1>(m))));
        row_byte[s] = block_byte16<FMT>(m & 0xffffu);
        row_byte[s + 1] = block_byte16<FMT>(m >> 16);
      }
      row_max[s] = m;
    }
    if constexpr (SQUARE) {
      uint32_t m = max_u16x2(max_u16x2(row_max[0], row_max[2]), max_u16x2(row_max[4], row_max[6]));
      m = max_u16x2(m, m >> 16 | m << 16);
      m = max_u16x2_dpp<0x140>(max_u16x2_dpp<0x141>(max_u16x2_dpp<0x4e>(max_u16x2_dpp<0xb1>(m))));
      auto r = __builtin_amdgcn_permlane16_swap(m, m, false, false);
      m = max_u16x2(r[0], r[1]);
      r = __builtin_amdgcn_permlane32_swap(m, m, false, false);
      m = max_u16x2(r[0], r[1]);
      if ((tid & 63) == 0) part[wave] = m & 0xffffu;
    } else if (transposed) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        auto r = __builtin_amdgcn_permlane16_swap(col_max[q], col_max[q], false, false);
        col_max[q] = max_u16x2(r[0], r[1]);
        r = __builtin_amdgcn_permlane32_swap(col_max[q], col_max[q], false, false);
        col_max[q] = max_u16x2(r[0], r[1]);
      }
      if ((tid & 63) < 16)
        *reinterpret_cast<uint4 *>(part + wave * (kTile / 2) + cl / 2) = make_uint4(col_max[0], col_max[1], col_max[2], col_max[3]);
    }
  } else {
    float row_max[kRows], col_max[8], all = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) col_max[e] = 0.0f;
#pragma unroll
    for (int s = 0; s < kRows; ++s) {
      row_max[s] = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float a = __builtin_fabsf(v.f(s, e));
        if (!NORM) row_max[s] = nan_max(row_max[s], a);
        if (!SQUARE) col_max[e] = nan_max(col_max[e], a);
      }
      if constexpr (SQUARE)
        all = nan_max(all, row_max[s]);
      else if constexpr (!NORM)
        row_byte[s] = block_byte<FMT>(max_lanes16(row_max[s]));
    }
    if constexpr (SQUARE) {
      all = max_lanes_by16(max_lanes16(all));
      if ((tid & 63) == 0) part[wave] = __float_as_uint(all);
    } else if (transposed) {
#pragma unroll
      for (int e = 0; e < 8; ++e) col_max[e] = max_lanes_by16(col_max[e]);
      if ((tid & 63) < 16) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
          *reinterpret_cast<f32x4 *>(part + wave * kTile + cl + h * HI) = f32x4{col_max[4 * h], col_max[4 * h + 1], col_max[4 * h + 2], col_max[4 * h + 3]};
      }
    }
  }
  if (SQUARE || transposed) __syncthreads();
  if constexpr (SQUARE) {
    uint32_t byte;
    if constexpr (PACKED)
      byte = block_byte16<FMT>(max(max(part[0], part[1]), max(part[2], part[3])));
    else
      byte = block_byte<FMT>(nan_max(nan_max(__uint_as_float(part[0]), __uint_as_float(part[1])),
                                     nan_max(__uint_as_float(part[2]), __uint_as_float(part[3]))));
#pragma unroll
    for (int s = 0; s < 8; ++s) row_byte[s] = col_byte[s] = byte;
    if (tid == 0) {
      if (p.row.data != nullptr) p.row.exps[tr * p.row.ld_exps + tc] = uint8_t(byte);
      if (transposed) p.col.exps[tc * p.col.ld_exps + tr] = uint8_t(byte);
    }
  } else if (transposed) {
    if constexpr (PACKED) {
      uint32_t m[4] = {0u, 0u, 0u, 0u};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint4 o = *reinterpret_cast<const uint4 *>(part + k * (kTile / 2) + cl / 2);
        m[0] = max_u16x2(m[0], o.x), m[1] = max_u16x2(m[1], o.y), m[2] = max_u16x2(m[2], o.z), m[3] = max_u16x2(m[3], o.w);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) col_byte[e] = block_byte16<FMT>(e % 2 == 0 ? m[e / 2] & 0xffffu : m[e / 2] >> 16);
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        f32x4 m = *reinterpret_cast<const f32x4 *>(part + cl + h * HI);
#pragma unroll
        for (int k = 1; k < 4; ++k) {
          const f32x4 o = *reinterpret_cast<const f32x4 *>(part + k * kTile + cl + h * HI);
#pragma unroll
          for (int e = 0; e < 4; ++e) m[e] = nan_max(m[e], o[e]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) col_byte[4 * h + e] = block_byte<FMT>(m[e]);
      }
    }
    if (rg == 0) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (!EDGE || col_of(e) < cols) p.col.exps[(c0 + col_of(e)) * p.col.ld_exps + tr] = uint8_t(col_byte[e]);
    }
  }

  // Row-wise codes.
  if (!NORM && p.row.data != nullptr) {
#pragma unroll
    for (int s = 0; s < kRows; ++s) {
      const int row = rg * kRows + s;
      const float step = block_step(row_byte[s]);
      uint32_t q[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if constexpr (PACKED)
          q[h] = convert_bf16<FMT, true>(convert_bf16<FMT, false>(0u, v.w[s][2 * h], step), v.w[s][2 * h + 1], step);
        else
          q[h] = convert_f32<FMT, true>(convert_f32<FMT, false>(0u, v.f(s, 4 * h), v.f(s, 4 * h + 1), step), v.f(s, 4 * h + 2),
                                        v.f(s, 4 * h + 3), step);
      }
      if (EDGE && row >= rows) continue;
      uint8_t *dst = p.row.data + (r0 + row) * p.row.ld + c0 + cl;
      if (!EDGE || cl + HI + 4 <= cols) {
        if constexpr (BF16) {
          store_out(dst, u32x2_out{q[0], q[1]}, (how & kRowLines) != 0);
        } else {
          *reinterpret_cast<u32_out *>(dst) = q[0];
          *reinterpret_cast<u32_out *>(dst + HI) = q[1];
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (col_of(e) < cols) dst[col_of(e) - cl] = uint8_t(byte_of(q[e / 4], e % 4));
      }
      if (!SQUARE && cl == 0) p.row.exps[(r0 + row) * p.row.ld_exps + tc] = uint8_t(row_byte[s]);
    }
  }
  if (!transposed) return;

  // Transposed codes: the lane's eight rows of each of its columns.
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float step = block_step(col_byte[e]);
    uint32_t q[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int s = 4 * h;
      if constexpr (PACKED) {
        const uint32_t sel = e % 2 == 0 ? 0x05040100u : 0x07060302u;
        const uint32_t a = __builtin_amdgcn_perm(v.w[s + 1][e / 2], v.w[s][e / 2], sel), b = __builtin_amdgcn_perm(v.w[s + 3][e / 2], v.w[s + 2][e / 2], sel);
        q[h] = convert_bf16<FMT, true>(convert_bf16<FMT, false>(0u, a, step), b, step);
      } else {
        q[h] = convert_f32<FMT, true>(convert_f32<FMT, false>(0u, v.f(s, e), v.f(s + 1, e), step), v.f(s + 2, e), v.f(s + 3, e), step);
      }
    }
    *reinterpret_cast<uint2 *>(tile + turned(col_of(e), rg >> 1) + (rg & 1) * 8) = make_uint2(q[0], q[1]);
  }
  __syncthreads();
  const int chunk = tid & 7, left = rows - chunk * 16;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int c = (tid >> 3) + 32 * j;
    if (EDGE && c >= cols) continue;
    const uint4 w4 = *reinterpret_cast<const uint4 *>(tile + turned(c, chunk));
    uint8_t *dst = p.col.data + (c0 + c) * p.col.ld + r0 + chunk * 16;
    if (!EDGE || left >= 16) {
      store_out(dst, u32x4_out{w4.x, w4.y, w4.z, w4.w}, (how & kColLines) != 0);
    } else {
      const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (e < left) dst[e] = uint8_t(byte_of(w[e / 4], e % 4));
    }
  }
}

template <bool BF16, int FMT, bool SQUARE, bool NORM>
__global__ __launch_bounds__(kThreads) void block_cast_kernel(BlockCastParams p, int tiles_r, int tiles_c, int how) {
  __shared__ __attribute__((aligned(16))) uint8_t tile[kTile * kTile];
  __shared__ __attribute__((aligned(16))) uint32_t part[4 * kTile];
  const int id = how & kByXcd ? xcd_remap(int(blockIdx.x), tiles_r * tiles_c) : int(blockIdx.x);
  const int tr = id / tiles_c, tc = id % tiles_c;
  if (int64_t(tr + 1) * kTile <= p.rows && int64_t(tc + 1) * kTile <= p.cols)
    cast_tile<BF16, FMT, SQUARE, NORM, false>(p, tr, tc, how, tile, part);
  else
    cast_tile<BF16, FMT, SQUARE, NORM, true>(p, tr, tc, how, tile, part);
}

template <bool BF16, int FMT>
hipError_t launch_fmt(const BlockCastParams &p, hipStream_t s) {
  const int64_t tiles_r = (p.rows + kTile - 1) / kTile, tiles_c = (p.cols + kTile - 1) / kTile;
  const dim3 grid{unsigned(tiles_r * tiles_c)}, block(kThreads);
  // Rows of tiles that stay on one XCD: neighbours write one line of codes, or of bytes, to
  // its L2.  The cast of BF16 in both orders, MI355X, us, over all XCDs / so: where lines of
  // codes are shared, 8008 x 8040 93 / 86, 1500 x 4099 13.2 / 11.8; with whole lines 4096 x
  // 4096 16.7 / 18.4, 8192 x 8192 57.5 / 65.6, 16384 x 16384 252 / 258, but 4096 x 28672
  // 107 / 100, 8192 x 28672 203 / 195, 57344 x 8192 in square blocks 362 / 348.  Row-wise
  // only it is 36.9 / 38.8, FP32 8192 x 8192 87 / 93, a norm's values 8192 x 8192, right after
  // the kernel that wrote its input, 121 / 134 (with that kernel): not there.
  const bool lines = whole_lines(p.col) && (p.row.data == nullptr || whole_lines(p.row));
  const bool by_xcd = BF16 && p.col.data != nullptr && p.rstd == nullptr && (!lines || p.cols > 16384 || p.rows * p.cols > int64_t(1) << 28);
  const int how = (by_xcd ? kByXcd : 0) | (whole_lines(p.row) ? kRowLines : 0) | (whole_lines(p.col) ? kColLines : 0);
  const bool square = (p.row.data != nullptr ? p.row : p.col).row_shift != 0;
  if (p.rstd != nullptr) return klaunch(block_cast_kernel<BF16, FMT, false, true>, grid, block, 0, s, p, int(tiles_r), int(tiles_c), how);
  return square ? klaunch(block_cast_kernel<BF16, FMT, true, false>, grid, block, 0, s, p, int(tiles_r), int(tiles_c), how)
                : klaunch(block_cast_kernel<BF16, FMT, false, false>, grid, block, 0, s, p, int(tiles_r), int(tiles_c), how);
}

}  // namespace

hipError_t launch_block_cast(const BlockCastParams &p, hipStream_t s) {
  if (p.rows <= 0 || p.cols <= 0 || (p.row.data == nullptr && p.col.data == nullptr)) return hipSuccess;
  const int fmt = (p.row.data != nullptr ? p.row : p.col).fmt;
  if (p.in.bf16) return fmt == 0 ? launch_fmt<true, 0>(p, s) : launch_fmt<true, 1>(p, s);
  return fmt == 0 ? launch_fmt<false, 0>(p, s) : launch_fmt<false, 1>(p, s);
}

}  // namespace qe
