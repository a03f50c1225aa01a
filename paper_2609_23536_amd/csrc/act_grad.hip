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
// where separate passes would write and read dZ in 16 bits once more.  MI355X, a
// gated pair in 8 bits, BF16 gradients: 8192 x 28672 to codes 395 us (4.8 TB/s),
// 2048 x 14336 55 us (4.3), 4096 x 14336 to dense BF16 88 us (5.4); kept in BF16
// instead, 8192 x 28672 465 us (5.0).
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

typedef unsigned int u32x4_f32 __attribute__((ext_vector_type(4), aligned(4)));
typedef float f32x4_in __attribute__((ext_vector_type(4), aligned(4)));

// Eight values of a row as they are stored, zero where they do not exist.
template <bool BF16>
struct RawEight {
  u32x4_in w[BF16 ? 1 : 2];
};
// Eight saved values: BF16, or codes and the byte of their group.
template <int KIND>
struct RawSaved {
  RawEight<true> v;
};
template <>
struct RawSaved<kSavedI8> {
  u32x2_out w;
  uint32_t byte;
};

struct Eight {
  float v[8];
};

// Elements at .. at + 7; nv of them exist.  Loads are non-temporal: nothing here is read twice.
template <bool BF16, bool FULL>
__device__ __forceinline__ RawEight<BF16> load_raw(const void *base, int64_t at, int nv) {
  RawEight<BF16> r;
  if (FULL || nv == 8) {
    const char *p = static_cast<const char *>(base) + at * (BF16 ? 2 : 4);
#pragma unroll
    for (int i = 0; i < (BF16 ? 1 : 2); ++i) {
      if constexpr (BF16)
        r.w[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_in *>(p + 16 * i));
      else
        r.w[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_f32 *>(p + 16 * i));
    }
  } else {
#pragma unroll
    for (int i = 0; i < (BF16 ? 1 : 2); ++i) r.w[i] = u32x4_in{0u, 0u, 0u, 0u};
    if (nv > 0) {  // single elements, the last one again past it: no load waits for another
      uint32_t x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int64_t i = at + (e < nv ? e : nv - 1);
        x[e] = BF16 ? uint32_t(static_cast<const uint16_t *>(base)[i]) : static_cast<const uint32_t *>(base)[i];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t v = e < nv ? x[e] : 0u;
        if constexpr (BF16)
          r.w[0][e / 2] |= v << (16 * (e % 2));
        else
          r.w[e / 4][e % 4] = v;
      }
    }
  }
  return r;
}
template <bool BF16>
__device__ __forceinline__ Eight unpack(const RawEight<BF16> &r) {
  Eight x;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (BF16) {
      x.v[2 * e] = __uint_as_float(r.w[0][e] << 16);
      x.v[2 * e + 1] = __uint_as_float(r.w[0][e] & 0xffff0000u);
    } else {
      x.v[e] = __uint_as_float(r.w[0][e]);
      x.v[4 + e] = __uint_as_float(r.w[1][e]);
    }
  }
  return x;
}
template <int KIND, bool FULL>
__device__ __forceinline__ RawSaved<KIND> load_saved(const SavedRef &s, int64_t row, int64_t col, int nv) {
  RawSaved<KIND> r;
  if constexpr (KIND == kSavedBF16) {
    r.v = load_raw<true, FULL>(s.data, row * s.ld + col, nv);
  } else {
    const uint8_t *p = static_cast<const uint8_t *>(s.data) + row * s.ld + col;
    r.byte = FULL || nv > 0 ? s.exps[row * s.ld_exps + col / kSaveGroup] : 0u;
    if (FULL || nv == 8) {
      r.w = __builtin_nontemporal_load(reinterpret_cast<const u32x2_out *>(p));
    } else {
      r.w = u32x2_out{0u, 0u};
      if (nv > 0) {
        uint32_t x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = p[e < nv ? e : nv - 1];
#pragma unroll
        for (int e = 0; e < 8; ++e) r.w[e / 4] |= (e < nv ? x[e] : 0u) << (8 * (e % 4));
      }
    }
  }
  return r;
}
template <int KIND>
__device__ __forceinline__ Eight restore(const RawSaved<KIND> &r) {
  if constexpr (KIND == kSavedBF16) {
    return unpack(r.v);
  } else {
    const f32x4 a = restore4(r.w[0], r.byte), b = restore4(r.w[1], r.byte);
    return Eight{{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}};
  }
}

// Code stores, non-temporal or not; between empty asm, or the compiler would merge
// the two into one ordinary store.
__device__ __forceinline__ void store_codes2(uint8_t *dst, u32x2_out v, int nt) {
  if (nt) {
    asm volatile("");
    __builtin_nontemporal_store(v, reinterpret_cast<u32x2_out *>(dst));
    asm volatile("");
  } else {
    *reinterpret_cast<u32x2_out *>(dst) = v;
  }
}
__device__ __forceinline__ void store_codes4(uint8_t *dst, u32x4_out v, int nt) {
  if (nt) {
    asm volatile("");
    __builtin_nontemporal_store(v, reinterpret_cast<u32x4_out *>(dst));
    asm volatile("");
  } else {
    *reinterpret_cast<u32x4_out *>(dst) = v;
  }
}

// Row tiles whose columns the workgroups in flight share: rows and transposed
// rows are usually a multiple of 4 KB apart, so that tiles side by side in one
// row tile write all their transposed codes to a few memory channels.  8192 x
// 28672 gated, MI355X: 1 446 us, 8 451, 16 453, 32 397, 64 408; 2048 x 14336 (16
// row tiles) 55 with 1, 53 with all.
constexpr int kGroupRows = 32;

template <bool GATED, bool BF16, int KIND, int ROWS, int THREADS>
__global__ __launch_bounds__(THREADS) void act_grad_kernel(ActGradParams p, int tiles_r, int tiles_c, int nt) {
  constexpr int OUTS = GATED ? 2 : 1;
  constexpr int RS = THREADS / 16;          // rows per step
  constexpr int STEPS = ROWS / RS;
  constexpr int RPL = ROWS / 8;             // rows and columns per lane when transposing
  constexpr int CPL = kTile * 8 / THREADS;
  __shared__ __attribute__((aligned(16))) uint8_t tile[OUTS][ROWS * kTile];
  static_assert(sizeof(tile) >= RS / 2 * kTile * sizeof(float), "the column sums' staging fits in the tile");
  const int tid = threadIdx.x;
  // Tiles go down groups of kGroupRows row tiles, column after column.
  const int in_group = kGroupRows * tiles_c, group = int(blockIdx.x) / in_group, first = group * kGroupRows;
  const int height = min(tiles_r - first, kGroupRows), at = int(blockIdx.x) - group * in_group;
  const int rt = first + at % height;
  const int64_t r0 = int64_t(rt) * ROWS, c0 = int64_t(at / height) * kTile;
  const int rl = tid >> 4, cl = (tid & 15) * 8;
  const int64_t col = c0 + cl;
  const int nc = int(p.cols - col < 0 ? 0 : (p.cols - col > 8 ? 8 : p.cols - col));
  const bool codes = p.scale != nullptr;
  const float scale = codes ? *p.scale : 0.0f;
  const bool e4m3 = p.fmt == 0;  // uniform
  const float fmax = e4m3 ? 448.0f : 57344.0f;
  if (blockIdx.x == 0 && tid == 0 && codes && p.snapshot != nullptr) *p.snapshot = *p.scale_inv;
  float amax = 0.0f;
  float sums[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};

  // Steps go in groups whose loads are all in flight together; FULL: every
  // element of the tile exists.
  auto run = [&](auto act, auto full) {
    constexpr bool FULL = decltype(full)::value;
    constexpr int G = FULL ? (STEPS < 4 ? STEPS : 4) : 2;
#pragma unroll 1
    for (int s0 = 0; s0 < STEPS; s0 += G) {
      RawEight<BF16> dd_raw[G];
      RawSaved<KIND> z_raw[G], u_raw[GATED ? G : 1];
      int nvs[G];
#pragma unroll
      for (int q = 0; q < G; ++q) {
        const int64_t row = r0 + (s0 + q) * RS + rl;
        nvs[q] = FULL ? 8 : (row < p.rows ? nc : 0);
        dd_raw[q] = load_raw<BF16, FULL>(p.dd, row * p.ld_dd + col, nvs[q]);
        z_raw[q] = load_saved<KIND, FULL>(p.z, row, col, nvs[q]);
        if constexpr (GATED) u_raw[q] = load_saved<KIND, FULL>(p.u, row, col, nvs[q]);
      }
#pragma unroll
      for (int q = 0; q < G; ++q) {
        const int row_l = (s0 + q) * RS + rl;
        const int64_t row = r0 + row_l;
        const int nv = nvs[q];
        const Eight dd = unpack(dd_raw[q]), z = restore(z_raw[q]);
        Eight u, d[OUTS];
        if constexpr (GATED) u = restore(u_raw[q]);
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
        if (!FULL && nv < 8) {  // a NaN in a group's exponent reaches the columns past the last one
#pragma unroll
          for (int o = 0; o < OUTS; ++o)
#pragma unroll
            for (int e = 0; e < 8; ++e) d[o].v[e] = e < nv ? d[o].v[e] : 0.0f;
        }
#pragma unroll
        for (int o = 0; o < OUTS; ++o) {
          const int64_t oc = col + (o == 0 ? 0 : p.cols);
          const float *v = d[o].v;
          float most = nan_max(amax4(f32x4{v[0], v[1], v[2], v[3]}), amax4(f32x4{v[4], v[5], v[6], v[7]}));
          amax = nan_max(amax, most);
          if constexpr (!GATED) {
#pragma unroll
            for (int e = 0; e < 8; ++e) sums[e] += v[e];
          }
          if (codes) {
            const float s8[8] = {v[0] * scale, v[1] * scale, v[2] * scale, v[3] * scale,
                                 v[4] * scale, v[5] * scale, v[6] * scale, v[7] * scale};
            uint32_t w0, w1;
            if (__builtin_expect(most * scale <= fmax, 1)) {
              w0 = e4m3 ? enc4_in_range<0>(s8[0], s8[1], s8[2], s8[3]) : enc4_in_range<1>(s8[0], s8[1], s8[2], s8[3]);
              w1 = e4m3 ? enc4_in_range<0>(s8[4], s8[5], s8[6], s8[7]) : enc4_in_range<1>(s8[4], s8[5], s8[6], s8[7]);
            } else {  // a value to saturate, or a NaN
              w0 = e4m3 ? enc4<0>(s8[0], s8[1], s8[2], s8[3]) : enc4<1>(s8[0], s8[1], s8[2], s8[3]);
              w1 = e4m3 ? enc4<0>(s8[4], s8[5], s8[6], s8[7]) : enc4<1>(s8[4], s8[5], s8[6], s8[7]);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                w0 = nan_fix(w0, e, v[e]);
                w1 = nan_fix(w1, e, v[4 + e]);
              }
            }
            *reinterpret_cast<uint2 *>(tile[o] + lds_chunk_offset<RPL>(row_l, cl >> 4) + (cl & 15)) = make_uint2(w0, w1);
            if (p.q_row != nullptr) {
              uint8_t *dst = p.q_row + row * p.ld_row + oc;
              if (FULL || nv == 8) {
                store_codes2(dst, u32x2_out{w0, w1}, nt);
              } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                  if (e < nv) dst[e] = uint8_t(byte_of(e < 4 ? w0 : w1, e % 4));
              }
            }
          }
          if (p.dz == nullptr) continue;
          if (p.dz_bf16) {
            uint16_t *dst = static_cast<uint16_t *>(p.dz) + row * p.ld_dz + oc;
            u32x4_in w;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = bf16x2_bits(d[o].v[2 * e], d[o].v[2 * e + 1]);
            if (FULL || nv == 8) {
              *reinterpret_cast<u32x4_in *>(dst) = w;
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (e < nv) dst[e] = uint16_t(w[e / 2] >> (16 * (e % 2)));
            }
          } else {
            float *dst = static_cast<float *>(p.dz) + row * p.ld_dz + oc;
            if (FULL || nv == 8) {
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
  };
  const bool full = r0 + ROWS <= p.rows && c0 + kTile <= p.cols;
  act_switch(p.act, [&](auto act) {
    if (full)
      run(act, std::true_type{});
    else
      run(act, std::false_type{});
  });

  const uint32_t wave_max = update_wave_max(abs_bits(amax));
  if (codes && p.q_col != nullptr) {
    __syncthreads();  // the tile's codes are in LDS
    const int rb = tid & 7, cq = tid >> 3;
    const int64_t n = p.rows - (r0 + rb * RPL);  // rows of this lane's block that exist (or more)
#pragma unroll
    for (int o = 0; o < OUTS; ++o) {
      uint32_t w[CPL][RPL / 4];  // [column][four rows]
#pragma unroll
      for (int q = 0; q < RPL / 4; ++q) {
        uint32_t d[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint8_t *at = tile[o] + lds_chunk_offset<RPL>(rb * RPL + 4 * q + i, cq * CPL >> 4) + (cq * CPL & 15);
          if constexpr (CPL == 4)
            d[i] = *reinterpret_cast<const uint32_t *>(at);
          else
            d[i] = *reinterpret_cast<const uint16_t *>(at);
        }
        // 4 x 4 (4 x 2) bytes transposed: pairs of rows, then pairs of pairs
        const uint32_t a = __builtin_amdgcn_perm(d[1], d[0], 0x05010400u), b = __builtin_amdgcn_perm(d[3], d[2], 0x05010400u);
        w[0][q] = __builtin_amdgcn_perm(b, a, 0x05040100u);
        w[1][q] = __builtin_amdgcn_perm(b, a, 0x07060302u);
        if constexpr (CPL == 4) {
          const uint32_t c = __builtin_amdgcn_perm(d[1], d[0], 0x07030602u), f = __builtin_amdgcn_perm(d[3], d[2], 0x07030602u);
          w[2][q] = __builtin_amdgcn_perm(f, c, 0x05040100u);
          w[3][q] = __builtin_amdgcn_perm(f, c, 0x07060302u);
        }
      }
#pragma unroll
      for (int j = 0; j < CPL; ++j) {
        const int64_t c = c0 + CPL * cq + j;
        if (c >= p.cols || n <= 0) continue;
        uint8_t *dst = p.q_col + (c + (o == 0 ? 0 : p.cols)) * p.ld_col + r0 + rb * RPL;
        if (n >= RPL) {
          if constexpr (RPL == 16)
            store_codes4(dst, u32x4_out{w[j][0], w[j][1], w[j][2], w[j][3]}, nt);
          else
            store_codes2(dst, u32x2_out{w[j][0], w[j][1]}, nt);
        } else {
#pragma unroll
          for (int e = 0; e < RPL; ++e)
            if (e < n) dst[e] = uint8_t(byte_of(w[j][e / 4], e % 4));
        }
      }
    }
  }
  if (codes) {
    __syncthreads();  // the tile has been read: its first words take the waves' maxima
    uint32_t *red = reinterpret_cast<uint32_t *>(tile[0]);
    if ((tid & 63) == 0) red[tid >> 6] = wave_max;
    __syncthreads();
    if (tid == 0) {
      uint32_t a = red[0];
      for (int w = 1; w < THREADS / 64; ++w) a = red[w] > a ? red[w] : a;
      fold_amax(p.amax_accum, p.amax_slot, a);
    }
  }

  if (!GATED && p.partials != nullptr && p.rows > 0) {
    __syncthreads();  // the tile has been read
    float *col_sums = reinterpret_cast<float *>(tile[0]);  // [half the row lanes][128 columns]
    if (rl < RS / 2) {
#pragma unroll
      for (int e = 0; e < 8; ++e) col_sums[rl * kTile + cl + e] = sums[e];
    }
    __syncthreads();
    if (rl >= RS / 2) {
#pragma unroll
      for (int e = 0; e < 8; ++e) col_sums[(rl - RS / 2) * kTile + cl + e] += sums[e];
    }
    __syncthreads();
    if (tid < kTile && c0 + tid < p.cols) {
      float a = 0.0f;
#pragma unroll
      for (int r = 0; r < RS / 2; ++r) a += col_sums[r * kTile + tid];
      p.partials[int64_t(rt) * p.cols + c0 + tid] = a;
    }
  }
}

// dbias[c] (=, or +=) the sum over row tiles of partials[t][c]: 64 columns a
// workgroup, four lanes a column, each every fourth tile, then those four; always
// in that order.
__global__ __launch_bounds__(kThreads) void bias_grad_kernel(const float *partials, float *dbias, int64_t tiles, int64_t cols,
                                                             int accumulate) {
  __shared__ float part[kThreads];
  const int64_t c = int64_t(blockIdx.x) * 64 + (threadIdx.x & 63);
  float a = 0.0f;
  if (c < cols) {
#pragma unroll 4
    for (int64_t t = threadIdx.x >> 6; t < tiles; t += 4) a += partials[t * cols + c];
  }
  part[threadIdx.x] = a;
  __syncthreads();
  if (threadIdx.x < 64 && c < cols) {
    a = (part[threadIdx.x] + part[64 + threadIdx.x]) + (part[128 + threadIdx.x] + part[192 + threadIdx.x]);
    dbias[c] = accumulate ? dbias[c] + a : a;
  }
}

template <bool GATED, bool BF16, int KIND>
hipError_t launch_rows(int rows_per_tile, const ActGradParams &p, hipStream_t s) {
  const bool empty = p.rows == 0 || p.cols == 0;  // one workgroup then writes the snapshot
  const int64_t tiles_r = empty ? 1 : (p.rows + rows_per_tile - 1) / rows_per_tile;
  const int64_t tiles_c = empty ? 1 : (p.cols + kTile - 1) / kTile;
  if (tiles_r * tiles_c >= int64_t(1) << 31) return hipErrorInvalidValue;
  // Codes that the 256 MB memory-side cache cannot keep until they are read are
  // stored non-temporally (8192 x 28672 gated, MI355X: 397 us without, 385 so).
  const int nt = p.rows * p.cols * (GATED ? 4 : 2) > (int64_t(256) << 20);
  const dim3 grid{unsigned(tiles_r * tiles_c)};
  return rows_per_tile == 64 ? klaunch(act_grad_kernel<GATED, BF16, KIND, 64, 512>, grid, dim3(512), 0, s, p, int(tiles_r), int(tiles_c), nt)
                             : klaunch(act_grad_kernel<GATED, BF16, KIND, 128, 256>, grid, dim3(256), 0, s, p, int(tiles_r), int(tiles_c), nt);
}

template <bool GATED>
hipError_t launch_kind(int rows, const ActGradParams &p, hipStream_t s) {
  if (p.z.kind == kSavedBF16)
    return p.dd_bf16 ? launch_rows<GATED, true, kSavedBF16>(rows, p, s) : launch_rows<GATED, false, kSavedBF16>(rows, p, s);
  return p.dd_bf16 ? launch_rows<GATED, true, kSavedI8>(rows, p, s) : launch_rows<GATED, false, kSavedI8>(rows, p, s);
}

}  // namespace

hipError_t launch_act_grad(const ActGradParams &p, float *dbias, bool accumulate, hipStream_t s) {
  // Up to four tiles of 128 rows a unit (what its registers hold) the tiles take 64
  // rows and twice the lanes: shorter chains, more waves to overlap them.
  // MI355X, us with 128 / 64 rows: gated 1024 x 14336 (896 tiles) 31.3 / 29.2, 4096 x 4096
  // (1024) 34.8 / 33.1, 1000 x 9000 FP32 with dense values and bias (568) 38.0 / 30.4;
  // beyond, the shorter runs of transposed codes cost more: 2048 x 10240 (1280) 59.2 /
  // 63.3, 2048 x 14336 (1792) 54.5 / 59.8.
  const int rows = ((p.rows + 127) / 128) * ((p.cols + kTile - 1) / kTile) <= 4 * compute_units() ? 64 : 128;
  if ((p.rows > 0 && p.cols > 0) || p.snapshot != nullptr) {
    const hipError_t e = p.u.kind != kSavedNone ? launch_kind<true>(rows, p, s) : launch_kind<false>(rows, p, s);
    if (e != hipSuccess) return e;
  }
  if (dbias == nullptr || p.cols <= 0) return hipSuccess;
  const int64_t tiles = (p.rows + rows - 1) / rows, blocks = (p.cols + 63) / 64;
  if (blocks >= int64_t(1) << 31) return hipErrorInvalidValue;
  return klaunch(bias_grad_kernel, dim3(unsigned(blocks)), dim3(kThreads), 0, s, p.partials, dbias, tiles, p.cols,
                 accumulate ? 1 : 0);
}

}  // namespace qe
