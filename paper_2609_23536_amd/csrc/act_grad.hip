// Gradient through an activation, from what the forward saved (gfx950):
//     dZ = dD * act'(Z)                                   one saved tensor
//     dG = dD * U * act'(G),  dU = dD * act(G)            a gated pair, side by side
// emitted as what the backward products read: FP8 codes row-wise (dI) and
// transposed (dW) at the role's delayed scale, with max |dZ| folded into its
// amax; optionally the dense values, and the column sums (the bias gradient).
// Values between the loads and the one rounding of each output are FP32.
//
// HBM-bound: per element it reads dD (2 or 4 bytes) and the saved values (33/32
// or 2 bytes each) and writes two code bytes per output (and the dense value),
// where separate passes would write and read dZ in 16 bits once more.
//
// Layout as in the cast (quantize.hip): a workgroup takes a tile of ROWS rows x
// 128 columns, a lane eight columns of every sixteenth row, so a saved group of
// 32 columns is four neighbouring lanes and every row run is a whole 128-byte
// line of codes; the codes are transposed through LDS.  Column sums: a lane's rows,
// then the sixteen lanes of a column through LDS, in a fixed order, to one partial
// sum per row tile; a second kernel adds those up in order.  So no result depends on
// the order of workgroups.
#include "act.h"
#include "scale_update.h"

namespace qe {
namespace {

typedef float f32x4_in __attribute__((ext_vector_type(4), aligned(4)));

struct Eight {
  float v[8];
};

// Values at .. at + 7 of a row, of which nv exist (the others read as zero).
__device__ __forceinline__ Eight load_bf16(const void *base, int64_t at, int nv) {
  Eight r;
  const uint16_t *p = static_cast<const uint16_t *>(base) + at;
  if (nv == 8) {
    const u32x4_in w = *reinterpret_cast<const u32x4_in *>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      r.v[2 * e] = __uint_as_float(w[e] << 16);
      r.v[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) r.v[e] = e < nv ? bf16_to_f32(p[e]) : 0.0f;
  }
  return r;
}
__device__ __forceinline__ Eight load_f32(const void *base, int64_t at, int nv) {
  Eight r;
  const float *p = static_cast<const float *>(base) + at;
  if (nv == 8) {
    const f32x4_in a = *reinterpret_cast<const f32x4_in *>(p), b = *reinterpret_cast<const f32x4_in *>(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      r.v[e] = a[e];
      r.v[4 + e] = b[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) r.v[e] = e < nv ? p[e] : 0.0f;
  }
  return r;
}
// Eight columns from `col` of row `row`, restored.
template <int KIND>
__device__ __forceinline__ Eight load_saved(const SavedRef &s, int64_t row, int64_t col, int nv) {
  if constexpr (KIND == kSavedBF16) {
    return load_bf16(s.data, row * s.ld + col, nv);
  } else {
    const uint8_t *p = static_cast<const uint8_t *>(s.data) + row * s.ld + col;
    u32x2_out w = {0u, 0u};
    uint32_t byte = 0u;
    if (nv == 8) {
      w = *reinterpret_cast<const u32x2_out *>(p);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < nv) w[e / 4] |= uint32_t(p[e]) << (8 * (e % 4));
    }
    if (nv > 0) byte = s.exps[row * s.ld_exps + col / kSaveGroup];
    const f32x4 a = restore4(w[0], byte), b = restore4(w[1], byte);
    return Eight{{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}};
  }
}

template <bool GATED, bool BF16, int KIND, int FMT, int ROWS>
__global__ __launch_bounds__(kThreads) void act_grad_kernel(ActGradParams p, int64_t tiles_c) {
  constexpr int OUTS = GATED ? 2 : 1;
  constexpr int STEPS = ROWS / 16;
  constexpr int RPL = ROWS / 8;  // rows per lane when transposing
  __shared__ __attribute__((aligned(16))) uint8_t tile[OUTS][ROWS * kTile];
  __shared__ uint32_t red[kThreads / 64];
  static_assert(sizeof(tile) >= 16 * kTile * sizeof(float), "the column sums' staging fits in the tile");
  const int tid = threadIdx.x;
  const int64_t rt = int64_t(blockIdx.x) / tiles_c;
  const int64_t r0 = rt * ROWS, c0 = int64_t(blockIdx.x) % tiles_c * kTile;
  const int rl = tid >> 4, cl = (tid & 15) * 8;
  const int64_t col = c0 + cl;
  const int nc = int(p.cols - col < 0 ? 0 : (p.cols - col > 8 ? 8 : p.cols - col));
  const bool codes = p.scale != nullptr;
  const float scale = codes ? *p.scale : 0.0f;
  if (blockIdx.x == 0 && tid == 0 && codes && p.snapshot != nullptr) *p.snapshot = *p.scale_inv;
  uint32_t amax = 0;
  float sums[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};

#pragma unroll 2
  for (int st = 0; st < STEPS; ++st) {
    const int row_l = st * 16 + rl;
    const int64_t row = r0 + row_l;
    const int nv = row < p.rows ? nc : 0;
    Eight dd, z, u;
    dd = BF16 ? load_bf16(p.dd, row * p.ld_dd + col, nv) : load_f32(p.dd, row * p.ld_dd + col, nv);
    z = load_saved<KIND>(p.z, row, col, nv);
    if constexpr (GATED) u = load_saved<KIND>(p.u, row, col, nv);
    Eight d[OUTS];
    act_switch(p.act, [&](auto act) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float v, slope;
        act_both<decltype(act)::value>(z.v[e], v, slope);
        if constexpr (GATED) {
          d[0].v[e] = dd.v[e] * u.v[e] * slope;
          d[1].v[e] = dd.v[e] * v;
        } else {
          d[0].v[e] = dd.v[e] * slope;
        }
      }
    });
    if (nv < 8) {  // a NaN in a group's exponent reaches the columns past the last one
#pragma unroll
      for (int o = 0; o < OUTS; ++o)
#pragma unroll
        for (int e = 0; e < 8; ++e) d[o].v[e] = e < nv ? d[o].v[e] : 0.0f;
    }
#pragma unroll
    for (int o = 0; o < OUTS; ++o) {
      const int64_t oc = col + (o == 0 ? 0 : p.cols);
      uint32_t most = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t b = abs_bits(d[o].v[e]);
        most = b > most ? b : most;
        if (!GATED) sums[e] += d[o].v[e];
      }
      amax = most > amax ? most : amax;
      if (codes) {
        const float *v = d[o].v;
        uint32_t w0 = enc4<FMT>(v[0] * scale, v[1] * scale, v[2] * scale, v[3] * scale);
        uint32_t w1 = enc4<FMT>(v[4] * scale, v[5] * scale, v[6] * scale, v[7] * scale);
        if (__builtin_expect(most > 0x7f800000u, 0)) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            w0 = nan_fix(w0, e, v[e]);
            w1 = nan_fix(w1, e, v[4 + e]);
          }
        }
        *reinterpret_cast<uint2 *>(tile[o] + lds_chunk_offset<RPL>(row_l, cl >> 4) + (cl & 15)) = make_uint2(w0, w1);
        if (p.q_row != nullptr) {
          uint8_t *dst = p.q_row + row * p.ld_row + oc;
          if (nv == 8) {
            *reinterpret_cast<u32x2_out *>(dst) = u32x2_out{w0, w1};
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (e < nv) dst[e] = uint8_t(byte_of(e < 4 ? w0 : w1, e % 4));
          }
        }
      }
      if (p.dz != nullptr) {
        if (p.dz_bf16) {
          uint16_t *dst = static_cast<uint16_t *>(p.dz) + row * p.ld_dz + oc;
          u32x4_in w;
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = bf16x2_bits(d[o].v[2 * e], d[o].v[2 * e + 1]);
          if (nv == 8) {
            *reinterpret_cast<u32x4_in *>(dst) = w;
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (e < nv) dst[e] = uint16_t(w[e / 2] >> (16 * (e % 2)));
          }
        } else {
          float *dst = static_cast<float *>(p.dz) + row * p.ld_dz + oc;
          if (nv == 8) {
            *reinterpret_cast<f32x4_in *>(dst) = f32x4_in{d[o].v[0], d[o].v[1], d[o].v[2], d[o].v[3]};
            *reinterpret_cast<f32x4_in *>(dst + 4) = f32x4_in{d[o].v[4], d[o].v[5], d[o].v[6], d[o].v[7]};
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (e < nv) dst[e] = d[o].v[e];
          }
        }
      }
    }
  }

  if (codes) {
    amax = update_wave_max(amax);
    if ((tid & 63) == 0) red[tid >> 6] = amax;
    __syncthreads();  // also: the tile's codes are in LDS
    if (tid == 0) {
      uint32_t a = red[0];
      for (int w = 1; w < kThreads / 64; ++w) a = red[w] > a ? red[w] : a;
      fold_amax(p.amax_accum, p.amax_slot, a);
    }
    if (p.q_col != nullptr) {
      const int rb = tid & 7, cq = tid >> 3;
      const int64_t n = p.rows - (r0 + rb * RPL);  // rows of this lane's block that exist (or more)
#pragma unroll
      for (int o = 0; o < OUTS; ++o) {
        uint32_t d[RPL];
#pragma unroll
        for (int i = 0; i < RPL; ++i)
          d[i] = *reinterpret_cast<const uint32_t *>(tile[o] + lds_chunk_offset<RPL>(rb * RPL + i, cq >> 2) + ((cq & 3) << 2));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int64_t c = c0 + 4 * cq + j;
          if (c >= p.cols || n <= 0) continue;
          uint32_t w[RPL / 4];
#pragma unroll
          for (int q = 0; q < RPL / 4; ++q)
            w[q] = byte_of(d[4 * q], j) | (byte_of(d[4 * q + 1], j) << 8) | (byte_of(d[4 * q + 2], j) << 16) |
                   (byte_of(d[4 * q + 3], j) << 24);
          uint8_t *dst = p.q_col + (c + (o == 0 ? 0 : p.cols)) * p.ld_col + r0 + rb * RPL;
          if (n >= RPL) {
            if constexpr (RPL == 16)
              *reinterpret_cast<u32x4_out *>(dst) = u32x4_out{w[0], w[1], w[2], w[3]};
            else
              *reinterpret_cast<u32x2_out *>(dst) = u32x2_out{w[0], w[1]};
          } else {
#pragma unroll
            for (int e = 0; e < RPL; ++e)
              if (e < n) dst[e] = uint8_t(byte_of(w[e / 4], e % 4));
          }
        }
      }
    }
  }

  if (!GATED && p.partials != nullptr && p.rows > 0) {
    __syncthreads();  // the tile has been read
    float *col_sums = reinterpret_cast<float *>(tile[0]);  // [16 row lanes][128 columns]
#pragma unroll
    for (int e = 0; e < 8; ++e) col_sums[rl * kTile + cl + e] = sums[e];
    __syncthreads();
    if (tid < kTile && c0 + tid < p.cols) {
      float a = 0.0f;
#pragma unroll
      for (int r = 0; r < 16; ++r) a += col_sums[r * kTile + tid];
      p.partials[rt * p.cols + c0 + tid] = a;
    }
  }
}

// dbias[c] (=, or +=) the sum over row tiles of partials[t][c], in order.
__global__ __launch_bounds__(kThreads) void bias_grad_kernel(const float *partials, float *dbias, int64_t tiles, int64_t cols,
                                                             int accumulate) {
  const int64_t c = int64_t(blockIdx.x) * kThreads + threadIdx.x;
  if (c >= cols) return;
  float a = 0.0f;
  for (int64_t t = 0; t < tiles; ++t) a += partials[t * cols + c];
  dbias[c] = accumulate ? dbias[c] + a : a;
}

template <bool GATED, bool BF16, int KIND, int FMT>
hipError_t launch_rows(int rows_per_tile, const ActGradParams &p, hipStream_t s) {
  const bool empty = p.rows == 0 || p.cols == 0;  // one workgroup then writes the snapshot
  const int64_t tiles_c = empty ? 1 : (p.cols + kTile - 1) / kTile;
  const int64_t tiles = empty ? 1 : (p.rows + rows_per_tile - 1) / rows_per_tile * tiles_c;
  if (tiles >= int64_t(1) << 31) return hipErrorInvalidValue;
  const dim3 grid{unsigned(tiles)}, block(kThreads);
  return rows_per_tile == 64 ? klaunch(act_grad_kernel<GATED, BF16, KIND, FMT, 64>, grid, block, 0, s, p, tiles_c)
                             : klaunch(act_grad_kernel<GATED, BF16, KIND, FMT, 128>, grid, block, 0, s, p, tiles_c);
}

template <bool GATED, bool BF16, int KIND>
hipError_t launch_fmt(int rows, const ActGradParams &p, hipStream_t s) {
  return p.fmt == 0 ? launch_rows<GATED, BF16, KIND, 0>(rows, p, s) : launch_rows<GATED, BF16, KIND, 1>(rows, p, s);
}

template <bool GATED>
hipError_t launch_kind(int rows, const ActGradParams &p, hipStream_t s) {
  if (p.z.kind == kSavedBF16)
    return p.dd_bf16 ? launch_fmt<GATED, true, kSavedBF16>(rows, p, s) : launch_fmt<GATED, false, kSavedBF16>(rows, p, s);
  return p.dd_bf16 ? launch_fmt<GATED, true, kSavedI8>(rows, p, s) : launch_fmt<GATED, false, kSavedI8>(rows, p, s);
}

}  // namespace

hipError_t launch_act_grad(const ActGradParams &p, float *dbias, bool accumulate, hipStream_t s) {
  const int rows = ((p.rows + 127) / 128) * ((p.cols + kTile - 1) / kTile) <= 512 ? 64 : 128;  // as the cast
  if ((p.rows > 0 && p.cols > 0) || p.snapshot != nullptr) {
    const hipError_t e = p.u.kind != kSavedNone ? launch_kind<true>(rows, p, s) : launch_kind<false>(rows, p, s);
    if (e != hipSuccess) return e;
  }
  if (dbias == nullptr || p.cols <= 0) return hipSuccess;
  const int64_t tiles = (p.rows + rows - 1) / rows, blocks = (p.cols + kThreads - 1) / kThreads;
  if (blocks >= int64_t(1) << 31) return hipErrorInvalidValue;
  return klaunch(bias_grad_kernel, dim3(unsigned(blocks)), dim3(kThreads), 0, s, p.partials, dbias, tiles, p.cols,
                 accumulate ? 1 : 0);
}

}  // namespace qe
