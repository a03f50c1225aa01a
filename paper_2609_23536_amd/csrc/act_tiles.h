// Tiles of FP8 products whose epilogue goes on past the sum, as device functions
// (gfx950): the kernels of act_gemm.hip (operands of one scale each) and
// block_gemm.hip (a scale for each block of 128) are calls of them.  act_gemm.hip
// describes what they compute and how.
#pragma once

#include "act.h"
#include "gemm_loops.h"

namespace qe {
namespace {

typedef unsigned int u32_at1 __attribute__((aligned(1)));
typedef uint16_t u16_at1 __attribute__((aligned(1)));
typedef unsigned int u32x4_at16 __attribute__((ext_vector_type(4)));
typedef float f32x4_at4 __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned int u32x2_at2 __attribute__((ext_vector_type(2), aligned(2)));

// Four values from row-major storage of either type; nv of them exist.  (Where
// some do not, the last one is read again: no load waits for another.)
__device__ __forceinline__ v4f load_quad(const void *base, bool bf16, int64_t at, int nv) {
  v4f r = {0.f, 0.f, 0.f, 0.f};
  if (bf16) {
    const uint16_t *p = static_cast<const uint16_t *>(base) + at;
    if (nv == 4) {
      const u32x2_at2 w = *reinterpret_cast<const u32x2_at2 *>(p);
      r = v4f{__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16),
              __uint_as_float(w.y & 0xffff0000u)};
    } else if (nv > 0) {
      r = v4f{bf16_to_f32(p[0]), bf16_to_f32(p[nv > 1 ? 1 : 0]), bf16_to_f32(p[nv - 1]), 0.f};
    }
  } else {
    const float *p = static_cast<const float *>(base) + at;
    if (nv == 4)
      r = *reinterpret_cast<const f32x4_at4 *>(p);
    else if (nv > 0)
      r = v4f{p[0], p[nv > 1 ? 1 : 0], p[nv - 1], 0.f};
  }
  return r;
}

__device__ __forceinline__ void store_quad(void *base, bool bf16, int64_t at, int nv, v4f v) {
  if (bf16) {
    const uint32_t lo = bf16x2_bits(v[0], v[1]), hi = bf16x2_bits(v[2], v[3]);
    uint16_t *p = static_cast<uint16_t *>(base) + at;
    if (nv == 4) {
      *reinterpret_cast<u32x2_at2 *>(p) = u32x2_at2{lo, hi};
    } else {
      if (nv > 0) p[0] = uint16_t(lo);
      if (nv > 1) p[1] = uint16_t(lo >> 16);
      if (nv > 2) p[2] = uint16_t(hi);
    }
  } else {
    float *p = static_cast<float *>(base) + at;
    if (nv == 4) {
      *reinterpret_cast<f32x4_at4 *>(p) = f32x4_at4{v[0], v[1], v[2], v[3]};
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (e < nv) p[e] = v[e];
    }
  }
}

// Saves a quad of row `row`, columns col .. col + 3 (nv of them exist, none on
// a row that is not `live`).  All eight lanes of a 32-column group are here
// together, with col a multiple of 4.
__device__ __forceinline__ void save_quad(const SavedRef &s, int64_t row, int64_t col, int nv, v4f z) {
  if (s.kind == kSavedBF16) {
    store_quad(s.data, true, row * s.ld + col, nv, z);
    return;
  }
  if (nv < 4) {
#pragma unroll
    for (int e = 0; e < 4; ++e) z[e] = e < nv ? z[e] : 0.0f;
  }
  const uint32_t byte = save_exponent(max_lanes8(amax4(z)));
  const uint32_t codes = __builtin_expect(save_rare(byte), 0) ? save_codes<true>(z, byte) : save_codes<false>(z, byte);
  uint8_t *p = static_cast<uint8_t *>(s.data) + row * s.ld + col;
  if (nv == 4) {
    *reinterpret_cast<u32_at1 *>(p) = codes;
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < nv) p[e] = uint8_t(codes >> (8 * e));
  }
  if (nv > 0 && (col & (kSaveGroup - 1)) == 0) s.exps[row * s.ld_exps + col / kSaveGroup] = uint8_t(byte);
}

// Sums of ROWS output rows from row0, OW outputs each from column col0, staged
// in LDS as rows of EP floats (gated: 16 gates, the same outputs' 16 ups, ..),
// finished and stored by LANES lanes, this one being lane `t`.
// FULL: all of them exist.
template <bool GATED, bool FULL, int ROWS, int OW, int LANES, int EP>
__device__ __forceinline__ void finish_some(const ActGemmParams &g, const float *ep, int t, int64_t row0, int64_t col0) {
  constexpr int LPR = OW / 4;              // lanes per row
  constexpr int RS = LANES / LPR;          // rows per step
  constexpr int STEPS = ROWS / RS;
  constexpr int Q = STEPS < 8 ? STEPS : 8;  // steps whose loads are in flight together
  // (OW = 16, half a saved group, only where nothing is saved in 8 bits)
  static_assert(OW % 16 == 0 && LANES % LPR == 0 && ROWS % RS == 0 && STEPS % Q == 0, "whole steps");
  const int rl = t / LPR, cl = (t % LPR) * 4;
  const int64_t col = col0 + cl;
  const int nv = FULL ? 4 : int(g.n - col < 0 ? 0 : (g.n - col > 4 ? 4 : g.n - col));
  const float *src = ep + rl * EP + (GATED ? (cl / 16) * 32 + cl % 16 : cl);
  v4f bias = {0.f, 0.f, 0.f, 0.f};
  if (!GATED && g.bias != nullptr) bias = load_quad(g.bias, g.bias_bf16 != 0, col, nv);
#pragma unroll 1
  for (int s0 = 0; s0 < STEPS; s0 += Q) {
    v4f z[Q], u[Q], r[Q];
    int live[Q];  // columns of the step that exist
#pragma unroll
    for (int q = 0; q < Q; ++q) live[q] = FULL || row0 + rl + (s0 + q) * RS < g.m ? nv : 0;
    if (!GATED && g.residual != nullptr) {
#pragma unroll
      for (int q = 0; q < Q; ++q)
        r[q] = load_quad(g.residual, g.residual_bf16 != 0, (row0 + rl + (s0 + q) * RS) * g.ld_residual + col, live[q]);
    }
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      z[q] = *reinterpret_cast<const v4f *>(src + (s0 + q) * (RS * EP)) + bias;
      if constexpr (GATED) u[q] = *reinterpret_cast<const v4f *>(src + (s0 + q) * (RS * EP) + 16);
    }
    if (g.z.kind != kSavedNone) {
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        save_quad(g.z, row0 + rl + (s0 + q) * RS, col, live[q], z[q]);
        if constexpr (GATED) save_quad(g.u, row0 + rl + (s0 + q) * RS, col, live[q], u[q]);
      }
    }
    act_switch(g.act, [&](auto act) {
#pragma unroll
      for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e) z[q][e] = act_value<decltype(act)::value>(z[q][e]);
    });
    if constexpr (GATED) {
#pragma unroll
      for (int q = 0; q < Q; ++q) z[q] *= u[q];
    } else if (g.residual != nullptr) {
#pragma unroll
      for (int q = 0; q < Q; ++q) z[q] += r[q];
    }
#pragma unroll
    for (int q = 0; q < Q; ++q)
      store_quad(g.c, g.c_bf16 != 0, (row0 + rl + (s0 + q) * RS) * g.ldc + col, live[q], z[q]);
  }
}

template <bool GATED, int ROWS, int OW, int LANES, int EP>
__device__ __forceinline__ void finish_rows(const ActGemmParams &g, const float *ep, int t, int64_t row0, int64_t col0) {
  if (row0 + ROWS <= g.m && col0 + OW <= g.n)
    finish_some<GATED, true, ROWS, OW, LANES, EP>(g, ep, t, row0, col0);
  else
    finish_some<GATED, false, ROWS, OW, LANES, EP>(g, ep, t, row0, col0);
}

// f(0), f(1), .. f(N - 1) as constants: accumulators indexed by a loop variable
// that is left in the code would go to memory.
template <int N, typename F>
__device__ __forceinline__ void static_for(F &&f) {
  if constexpr (N > 0) {
    static_for<N - 1>(f);
    f(std::integral_constant<int, N - 1>{});
  }
}

// A wave's block of 16 NR rows x 16 QUADS columns, of which the lane holds quad q
// of rows 16 h + (lane & 15): columns 16 q + 4 (lane >> 4) ..  It goes through
// LDS, so that the lanes then write whole row runs, 16 bytes each (LDS operations
// of one wave complete in order).  Rows of RUN bytes, PITCH apart in LDS.
template <int QUADS, int ES>
struct Rows {
  static constexpr int RUN = 16 * QUADS * ES, PITCH = RUN + 16, LPR = RUN / 16, RS = 64 / LPR;  // lanes a row, rows a step
};

template <int QUADS, int NR, bool BF16>
__device__ __forceinline__ void stage_block(uint8_t *ls, int lane, const v4f (&v)[NR][QUADS]) {
  using L = Rows<QUADS, BF16 ? 2 : 4>;
#pragma unroll
  for (int h = 0; h < NR; ++h)
#pragma unroll
    for (int q = 0; q < QUADS; ++q) {
      uint8_t *at = ls + (16 * h + (lane & 15)) * L::PITCH + (16 * q + 4 * (lane >> 4)) * (BF16 ? 2 : 4);
      if constexpr (BF16)
        *reinterpret_cast<uint2 *>(at) = make_uint2(bf16x2_bits(v[h][q][0], v[h][q][1]), bf16x2_bits(v[h][q][2], v[h][q][3]));
      else
        *reinterpret_cast<v4f *>(at) = v[h][q];
    }
}

// Codes of an 8-bit checkpoint (a group is two quads of four lanes), and the exponent
// bytes straight to memory, from lanes 0 .. 15 of each block row.
template <bool EDGE, int QUADS, int NR>
__device__ __forceinline__ void stage_codes(uint8_t *ls, int lane, uint8_t *exps, int64_t ld_exps, int rows, int cols,
                                            const v4f (&v)[NR][QUADS]) {
  using L = Rows<QUADS, 1>;
  static_assert(QUADS == 4 || QUADS == 8, "whole groups, their bytes in a word");
  uint32_t byte[NR][QUADS / 2], most = 0u;
#pragma unroll
  for (int h = 0; h < NR; ++h)
#pragma unroll
    for (int q = 0; q < QUADS / 2; ++q) {
      byte[h][q] = save_exponent(max_lanes_by16(nan_max(amax4(v[h][2 * q]), amax4(v[h][2 * q + 1]))));
      most = byte[h][q] > most ? byte[h][q] : most;
    }
  auto codes = [&](auto rare) {
    constexpr bool RARE = decltype(rare)::value;
#pragma unroll
    for (int h = 0; h < NR; ++h)
#pragma unroll
      for (int q = 0; q < QUADS; ++q)
        *reinterpret_cast<uint32_t *>(ls + (16 * h + (lane & 15)) * L::PITCH + 16 * q + 4 * (lane >> 4)) =
            save_codes<RARE>(v[h][q], byte[h][q / 2]);
  };
  if (__builtin_expect(save_rare(most), 0))
    codes(std::true_type{});
  else
    codes(std::false_type{});
#pragma unroll
  for (int h = 0; h < NR; ++h) {
    uint32_t bytes = 0u;
#pragma unroll
    for (int q = 0; q < QUADS / 2; ++q) bytes |= byte[h][q] << (8 * q);
    if (lane < 16 && (!EDGE || 16 * h + lane < rows)) {
      uint8_t *at = exps + (16 * h + lane) * ld_exps;
      if (EDGE && cols < 16 * QUADS) {
#pragma unroll
        for (int q = 0; q < QUADS / 2; ++q)
          if (q * kSaveGroup < cols) at[q] = uint8_t(bytes >> (8 * q));
      } else if constexpr (QUADS == 8) {
        *reinterpret_cast<u32_out *>(at) = bytes;
      } else {
        *reinterpret_cast<u16_at1 *>(at) = uint16_t(bytes);
      }
    }
  }
}

// The staged block to memory: `base` is its first element, `pitch` in bytes.
// EDGE: rows x cols of it exist.
template <bool EDGE, int QUADS, int NR, int ES>
__device__ __forceinline__ void store_staged(const uint8_t *ls, int lane, void *base, int64_t pitch, int rows, int cols) {
  using L = Rows<QUADS, ES>;
  char *out = static_cast<char *>(base) + (lane / L::LPR) * pitch + (lane % L::LPR) * 16;
  const uint8_t *in = ls + (lane / L::LPR) * L::PITCH + (lane % L::LPR) * 16;
#pragma unroll
  for (int s = 0; s < 16 * NR / L::RS; ++s) {
    const u32x4_at16 v = *reinterpret_cast<const u32x4_at16 *>(in + s * (L::RS * L::PITCH));
    char *dst = out + s * L::RS * pitch;
    if constexpr (EDGE) {
      const int n = (cols - lane % L::LPR * (16 / ES)) * ES;  // bytes of the lane's sixteen that exist
      if (s * L::RS + lane / L::LPR >= rows || n <= 0) continue;
      if (n < 16) {
#pragma unroll
        for (int b = 0; b < 16; b += ES) {
          if (b >= n) break;
          if constexpr (ES == 1) dst[b] = char(v[b / 4] >> (8 * (b % 4)));
          if constexpr (ES == 2) *reinterpret_cast<uint16_t *>(dst + b) = uint16_t(v[b / 4] >> (8 * (b % 4)));
          if constexpr (ES == 4) *reinterpret_cast<uint32_t *>(dst + b) = v[b / 4];
        }
        continue;
      }
    }
    __builtin_nontemporal_store(v, reinterpret_cast<u32x4_out *>(dst));
  }
}

// A lane's residual quads of a block row, as stored: from element `at`, `cols`
// of which exist.
template <bool EDGE, int QUADS>
struct Quads {
  v4f raw[QUADS];  // BF16: the first two words
  __device__ __forceinline__ void load(const void *base, bool bf16, int64_t at, int cols) {
#pragma unroll
    for (int j = 0; j < QUADS; ++j) {
      if (EDGE && cols < 16 * j + 4) {  // not the whole quad
        const v4f r = load_quad(base, bf16, at + 16 * j, max(cols - 16 * j, 0));
        raw[j] = r;
        if (bf16) {
          raw[j][0] = __uint_as_float(bf16x2_bits(r[0], r[1]));
          raw[j][1] = __uint_as_float(bf16x2_bits(r[2], r[3]));
        }
      } else if (bf16) {
        const u32x2_at2 w = *reinterpret_cast<const u32x2_at2 *>(static_cast<const uint16_t *>(base) + at + 16 * j);
        raw[j][0] = __uint_as_float(w.x);
        raw[j][1] = __uint_as_float(w.y);
      } else {
        raw[j] = *reinterpret_cast<const f32x4_at4 *>(static_cast<const float *>(base) + at + 16 * j);
      }
    }
  }
  __device__ __forceinline__ v4f get(bool bf16, int j) const {
    if (!bf16) return raw[j];
    const uint32_t a = __float_as_uint(raw[j][0]), b = __float_as_uint(raw[j][1]);
    return v4f{__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u), __uint_as_float(b << 16), __uint_as_float(b & 0xffff0000u)};
  }
};

__device__ __forceinline__ v4f scaled(v4f a, SumScale s) { return v4f{s(a[0]), s(a[1]), s(a[2]), s(a[3])}; }

struct TilePlace {
  int64_t m0, n0;  // first row, first output column
};

// The tile of this workgroup: the order of the plain GEMM (kGroupM, xcd_remap).
__device__ __forceinline__ TilePlace place(int tiles_m, int tiles_n, int bm, int bno) {
  const int pid = xcd_remap(blockIdx.x, tiles_m * tiles_n);
  const int in_group = kGroupM * tiles_n;
  const int first_m = pid / in_group * kGroupM;
  const int gsize = min(tiles_m - first_m, kGroupM);
  return {int64_t(first_m + (pid % in_group) % gsize) * bm, int64_t((pid % in_group) / gsize) * bno};
}

// An address that is the same in the whole wave, in scalar registers (the K
// loops' inline assembly takes it there; the compiler computes it in vector ones).
__device__ __forceinline__ const uint8_t *uniform(const uint8_t *p) {
  const uint64_t v = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(int(uint32_t(v))), hi = __builtin_amdgcn_readfirstlane(int(v >> 32));
  return reinterpret_cast<const uint8_t *>(uint64_t(hi) << 32 | lo);
}

// The scales of a tile's rows: one for each operand, applied to the sums, or a block's
// each, which the K loops take.
template <typename P>
constexpr bool kBlocked = std::is_base_of<BlockGemmParams, P>::value;
template <typename P>
__device__ __forceinline__ SumScale scale_of(const P &g, const float *b_inv) {
  if constexpr (kBlocked<P>)
    return {1.0f, 1.0f};
  else
    return sum_scale(g.a_scale_inv, b_inv);
}
template <int BM, int BN, int BUFS, typename P>
__device__ __forceinline__ auto tile_scales(const P &g, TilePlace at, uint32_t lds) {
  if constexpr (kBlocked<P>) {
    LdsScales<BM, BN, BUFS> sc;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int q = 0; q < sc.kPer; ++q) {
      const int slot = wave + 4 * q;
      const bool of_a = slot < BM / 64;
      const int64_t row0 = of_a ? at.m0 : at.n0, last = (of_a ? g.m : g.n) - 1, ld = of_a ? g.ld_a_exps : g.ld_b_exps;
      const int shift = of_a ? g.a_shift : g.b_shift;
      const int64_t row = min(row0 + (slot * 64 + lane - (of_a ? 0 : BM)), last);
      sc.base[q] = uniform((of_a ? g.a_exps : g.b_exps) + (row0 >> shift) * ld);
      sc.off[q] = uint32_t(((row >> shift) - (row0 >> shift)) * ld);
    }
    sc.groups = int((g.k + 4 * BK - 1) / (4 * BK));
    sc.lds = lds;
    return sc;
  } else {
    return NoScales{};
  }
}
template <typename P, int BM, int BN, int BUFS>
constexpr int kScaleBytes = kBlocked<P> ? LdsScales<BM, BN, BUFS>::kBytes : 0;

// Operand B of a tile: its base for this wave, and the B row (from n0) of LDS row r.
template <bool GATED>
__device__ __forceinline__ const uint8_t *b_base(const ActGemmParams &g, int64_t n0) {
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  return uniform((GATED && (wave & 2) != 0 ? g.b2 : g.b) + n0 * g.ldb);
}
template <bool GATED>
__device__ __forceinline__ int b_row(int r) {
  return GATED ? (r >> 5) * 16 + (r & 15) : r;
}

// Sums that are only rounded or added to a residual, of a whole wave's block of TM rows
// x 128 columns: 16 rows at a time through LDS and out in whole row runs, every address a
// scalar row offset and one of the lane's (with one wave a SIMD the instructions are the
// time).  The residual, of the output's type, is read in the order of the stores, 16 rows
// ahead.  RES: there may be one, `has` says whether (two variants of FP32 spill).  MI355X,
// us, block scales, by the general epilogue / so: BF16 6144 x 4096 x 2048 57 / 50, with a
// residual 78 / 59; 4096 x 14336 x 4096 210 / 191, with one 261 / 211.
template <int TM, bool BF16, bool RES>
__device__ __forceinline__ void store_sums(const ActGemmParams &g, const v4f (&acc)[TM / 16][8], uint8_t *ls, int lane, int64_t row0, int64_t col0,
                                           bool has) {
  constexpr int ES = BF16 ? 2 : 4;                                         // bytes an element
  constexpr int LPR = BF16 ? 16 : 32, STEP = 64 / LPR, STEPS = 16 / STEP;  // lanes a row, rows and steps
  constexpr bool NARROW = BF16 && !RES;                                    // rounded before the trip
  constexpr int PITCH = NARROW ? (128 + 8) * 2 : (128 + 4) * 4;
  auto rsrc = [&](const void *p, int64_t ld) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(uniform(static_cast<const uint8_t *>(p) + (row0 * ld + col0) * ES)), short(0), 0x7fffffff, 0x00020000);
  };
  const __amdgpu_buffer_rsrc_t out = rsrc(g.c, g.ldc), in = RES && has ? rsrc(g.residual, g.ld_residual) : out;
  const int pitch = int(g.ldc) * ES, in_pitch = int(g.ld_residual) * ES;
  const uint32_t at = uint32_t(lane / LPR) * uint32_t(pitch) + lane % LPR * 16, in_at = uint32_t(lane / LPR) * uint32_t(in_pitch) + lane % LPR * 16;
  v4i res[2][RES ? STEPS : 1] = {};
  auto fetch = [&](auto block) {
    constexpr int i = decltype(block)::value;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) res[i % 2][s] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(in, in_at, (16 * i + STEP * s) * in_pitch, kNT));
  };
  if constexpr (RES)
    if (has) fetch(std::integral_constant<int, 0>{});
  static_for<TM / 16>([&](auto block) {
    constexpr int i = decltype(block)::value;
    if constexpr (RES && i + 1 < TM / 16)
      if (has) fetch(std::integral_constant<int, i + 1>{});
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const v4f a = acc[i][j];
      uint8_t *to = ls + (lane & 15) * PITCH + (16 * j + 4 * (lane >> 4)) * (NARROW ? 2 : 4);
      if constexpr (NARROW)
        *reinterpret_cast<uint2 *>(to) = make_uint2(bf16x2_bits(a[0], a[1]), bf16x2_bits(a[2], a[3]));
      else
        *reinterpret_cast<v4f *>(to) = a;
    }
    // (LDS operations of one wave complete in order)
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const uint8_t *from = ls + (lane / LPR + STEP * s) * PITCH + lane % LPR * (128 / LPR) * (NARROW ? 2 : 4);
      v4i w;
      if constexpr (NARROW) {
        w = *reinterpret_cast<const v4i *>(from);
      } else {
        float f[128 / LPR];
#pragma unroll
        for (int q = 0; q < 32 / LPR; ++q) {
          const v4f v = *reinterpret_cast<const v4f *>(from + 16 * q);
#pragma unroll
          for (int e = 0; e < 4; ++e) f[4 * q + e] = v[e];
        }
#pragma unroll
        for (int e = 0; e < 128 / LPR; ++e)
          if constexpr (RES) {
            const uint32_t r = uint32_t(res[i % 2][s][BF16 ? e / 2 : e]);
            const float sum = f[e] + __uint_as_float(!BF16 ? r : (e % 2 == 0 ? r << 16 : r & 0xffff0000u));
            f[e] = has ? sum : f[e];
          }
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = BF16 ? int(bf16x2_bits(f[BF16 ? 2 * e : 0], f[BF16 ? 2 * e + 1 : 0])) : int(__float_as_uint(f[e]));
      }
      __builtin_amdgcn_raw_buffer_store_b128(w, out, at, (16 * i + STEP * s) * pitch, kNT);
    }
    __builtin_amdgcn_sched_barrier(0);
  });
}

// Whether a product's sums can go that way: no more than a residual of the output's type in
// the epilogue, rows of both aligned to four elements, and a tile's rows within 2^31 bytes.
__device__ __forceinline__ bool only_sums(const ActGemmParams &g, int rows) {
  const int es = g.c_bf16 ? 2 : 4;
  auto fits = [&](const void *p, int64_t ld) { return ld % 4 == 0 && uintptr_t(p) % (4 * es) == 0 && ld * es * (rows + 4) < int64_t(1) << 31; };
  return g.act == kActNone && g.bias == nullptr && g.z.kind == kSavedNone && fits(g.c, g.ldc) &&
         (g.residual == nullptr || ((g.residual_bf16 != 0) == (g.c_bf16 != 0) && fits(g.residual, g.ld_residual)));
}

// OUT: the output's type where the kernel is one type's, which then stores bare sums by
// store_sums.
enum TileOut { kEither, kF32, kBF16 };
template <bool GATED, int FA, int FB, int BM, int BN, TileOut OUT = kEither, typename P>
__device__ __forceinline__ void act_large_tile(const P &g, int tiles_m, int tiles_n) {
  constexpr int NW = 4, TM = BM / 2, TN = BN / 2, BNO = GATED ? BN / 2 : BN;
  constexpr int I = TM / 16, J = TN / 16;
  constexpr int CHA = BM / 32, CHB = BN / 32;
  constexpr int STAGE = (BM + BN) * BK;
  static_assert(J % 2 == 0 && I % 2 == 0, "block columns and rows in pairs");
  __shared__ __attribute__((aligned(16))) uint8_t smem[2 * STAGE + NW * 1024 + kScaleBytes<P, BM, BN, 2>];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const TilePlace at = place(tiles_m, tiles_n, BM, BNO);
  uint32_t oa[CHA], ob[CHB];
#pragma unroll
  for (int c = 0; c < CHA; ++c) {
    const int row = 8 * (wave + NW * c) + (lane >> 3);
    oa[c] = chunk_offset(min(int64_t(row), g.m - 1 - at.m0), g.lda, (lane & 7) ^ row_swizzle(row), g.k);
  }
#pragma unroll
  for (int c = 0; c < CHB; ++c) {
    const int row = 8 * (wave + NW * c) + (lane >> 3);
    ob[c] = chunk_offset(min(int64_t(b_row<GATED>(row)), g.n - 1 - at.n0), g.ldb, (lane & 7) ^ row_swizzle(row), g.k);
  }
  v4f acc[I][J];
  large_k_loop<FA, FB, BM, BN>(uniform(g.a + at.m0 * g.lda), b_base<GATED>(g, at.n0), oa, ob, g.k, smem, acc,
                               tile_scales<BM, BN, 2>(g, at, 2 * STAGE + NW * 1024));

  __syncthreads();  // every wave is done reading the last stage
  const int fr = lane & 15, fq = lane >> 4;
  const SumScale s0 = scale_of(g, g.b_scale_inv), s1 = GATED ? scale_of(g, g.b2_scale_inv) : s0;
  // A tile finishes in the accumulators' own layout, where a lane holds four
  // neighbouring outputs of one row (and their gates beside their ups), a block
  // of rows at a time; only what is stored goes through LDS.  The residual is
  // read in that layout too (32-byte pieces of BF16 rows, four of which share a
  // line while it is in the L1), before the block above it is stored: read row by
  // row when due it cost 37 us a round of tiles on MI355X, against 16 in all
  // without it.  (Bringing its lines into the L2 before the K loop: slower.)
  // Gated tiles take two block rows at a time (K = 256: one 79 us, two 74); plain
  // ones one, two spill.
  constexpr int QV = GATED ? J / 2 : J;  // quads a lane holds of an output row
  constexpr int NR = GATED ? 2 : 1;      // block rows at a time
  const int wu = __builtin_amdgcn_readfirstlane(wave);
  const int64_t wrow = at.m0 + (wu >> 1) * TM, wcol = at.n0 + (wu & 1) * (16 * QV);
  const int rows_left = int(min(int64_t(BM), g.m - wrow)), cols = int(min(int64_t(BN), g.n - wcol));  // of the wave's block, or more
  if (rows_left <= 0 || cols <= 0) return;
  uint8_t *ls = smem + wave * (STAGE / 2), *ls_u = ls + 16 * NR * Rows<QV, 2>::PITCH;
  uint8_t *ls_c = GATED ? ls_u + 16 * NR * Rows<QV, 2>::PITCH : ls_u;  // D last: at most FP32
  static_assert(16 * NR * ((GATED ? 2 : 1) * Rows<QV, 2>::PITCH + Rows<QV, 4>::PITCH) <= STAGE / 2, "the blocks staged fit");
  const bool has_res = !GATED && g.residual != nullptr, res_bf16 = g.residual_bf16 != 0;
  if constexpr (OUT != kEither) {
    static_assert(TN == 128 && !GATED, "blocks of 128 columns a wave");
    if (rows_left >= TM && cols >= TN && only_sums(g, TM)) {
      if (OUT == kBF16 && !has_res) return store_sums<TM, true, false>(g, acc, ls, lane, wrow, wcol, false);
      return store_sums<TM, OUT == kBF16, true>(g, acc, ls, lane, wrow, wcol, OUT == kBF16 || has_res);
    }
  }
  const bool i8 = g.z.kind == kSavedI8, kept = g.z.kind == kSavedBF16;
  auto finish = [&](auto edge) {
    constexpr bool EDGE = decltype(edge)::value;  // part of the wave's block does not exist
    v4f bias[QV];
    Quads<EDGE, QV> res;
    auto load_res = [&](int i) {
      const int64_t r = EDGE ? min(wrow + 16 * i + fr, g.m - 1) : wrow + 16 * i + fr;
      res.load(g.residual, res_bf16, r * g.ld_residual + wcol + 4 * fq, cols - 4 * fq);
    };
    if (has_res) load_res(0);
    if constexpr (!GATED) {
#pragma unroll
      for (int j = 0; j < QV; ++j) {
        bias[j] = v4f{0.f, 0.f, 0.f, 0.f};
        const int nv = EDGE ? max(0, min(4, cols - 16 * j - 4 * fq)) : 4;
        if (g.bias != nullptr) bias[j] = load_quad(g.bias, g.bias_bf16 != 0, wcol + 16 * j + 4 * fq, nv);
      }
    }
    static_for<I / NR>([&](auto block) {
      constexpr int i = decltype(block)::value * NR;
      const int64_t row = wrow + i * 16;
      const int rows = rows_left - i * 16;
      if (EDGE && rows <= 0) return;
      v4f z[NR][QV], up[NR][QV];
#pragma unroll
      for (int h = 0; h < NR; ++h)
#pragma unroll
        for (int j = 0; j < QV; ++j) {
          if constexpr (GATED) {
            z[h][j] = scaled(acc[i + h][2 * j], s0);
            up[h][j] = scaled(acc[i + h][2 * j + 1], s1);
          } else {
            z[h][j] = scaled(acc[i + h][j], s0) + bias[j];
          }
          if constexpr (EDGE) {  // columns past the last one count as zero in their group
            const int nv = cols - 16 * j - 4 * fq;
            z[h][j] = v4f{nv > 0 ? z[h][j][0] : 0.f, nv > 1 ? z[h][j][1] : 0.f, nv > 2 ? z[h][j][2] : 0.f, nv > 3 ? z[h][j][3] : 0.f};
            if constexpr (GATED)
              up[h][j] = v4f{nv > 0 ? up[h][j][0] : 0.f, nv > 1 ? up[h][j][1] : 0.f, nv > 2 ? up[h][j][2] : 0.f, nv > 3 ? up[h][j][3] : 0.f};
          }
        }
      if (i8) {
        stage_codes<EDGE, QV, NR>(ls, lane, g.z.exps + row * g.z.ld_exps + wcol / kSaveGroup, g.z.ld_exps, rows, cols, z);
        if constexpr (GATED)
          stage_codes<EDGE, QV, NR>(ls_u, lane, g.u.exps + row * g.u.ld_exps + wcol / kSaveGroup, g.u.ld_exps, rows, cols, up);
      } else if (kept) {
        stage_block<QV, NR, true>(ls, lane, z);
        if constexpr (GATED) stage_block<QV, NR, true>(ls_u, lane, up);
      }
      act_switch(g.act, [&](auto act) {
#pragma unroll
        for (int h = 0; h < NR; ++h)
#pragma unroll
          for (int j = 0; j < QV; ++j) {
            v4f d = z[h][j];
            if constexpr (GATED)
              d = v4f{act_value<decltype(act)::value>(d[0]) * up[h][j][0], act_value<decltype(act)::value>(d[1]) * up[h][j][1],
                      act_value<decltype(act)::value>(d[2]) * up[h][j][2], act_value<decltype(act)::value>(d[3]) * up[h][j][3]};
            else
              d = v4f{act_value<decltype(act)::value>(d[0]), act_value<decltype(act)::value>(d[1]),
                      act_value<decltype(act)::value>(d[2]), act_value<decltype(act)::value>(d[3])};
            z[h][j] = d;
          }
      });
      if (has_res) {
#pragma unroll
        for (int j = 0; j < QV; ++j) z[0][j] += res.get(res_bf16, j);
        if (i + 1 < I) load_res(i + 1);
      }
      // what was staged first has long been written when it is read back
      if (i8) {
        store_staged<EDGE, QV, NR, 1>(ls, lane, static_cast<uint8_t *>(g.z.data) + row * g.z.ld + wcol, g.z.ld, rows, cols);
        if constexpr (GATED)
          store_staged<EDGE, QV, NR, 1>(ls_u, lane, static_cast<uint8_t *>(g.u.data) + row * g.u.ld + wcol, g.u.ld, rows, cols);
      } else if (kept) {
        store_staged<EDGE, QV, NR, 2>(ls, lane, static_cast<uint16_t *>(g.z.data) + row * g.z.ld + wcol, g.z.ld * 2, rows, cols);
        if constexpr (GATED)
          store_staged<EDGE, QV, NR, 2>(ls_u, lane, static_cast<uint16_t *>(g.u.data) + row * g.u.ld + wcol, g.u.ld * 2, rows, cols);
      }
      if (OUT == kEither ? g.c_bf16 != 0 : OUT == kBF16) {
        stage_block<QV, NR, true>(ls_c, lane, z);
        store_staged<EDGE, QV, NR, 2>(ls_c, lane, static_cast<uint16_t *>(g.c) + row * g.ldc + wcol, g.ldc * 2, rows, cols);
      } else {
        stage_block<QV, NR, false>(ls_c, lane, z);
        store_staged<EDGE, QV, NR, 4>(ls_c, lane, static_cast<float *>(g.c) + row * g.ldc + wcol, g.ldc * 4, rows, cols);
      }
    });
  };
  if (rows_left >= TM && cols >= 16 * QV)
    finish(std::false_type{});
  else
    finish(std::true_type{});
}

template <bool GATED, int FA, int FB, int BM, int BN, int S, typename P>
__device__ __forceinline__ void act_ring_tile(const P &g, int tiles_m, int tiles_n) {
  constexpr int NW = 4, TM = BM / 2, TN = BN / 2, BNO = GATED ? BN / 2 : BN;
  constexpr int I = TM / 16, J = TN / 16;
  constexpr int CHA = BM / 32, CHB = BN / 32;
  constexpr int STAGE = (BM + BN) * BK;
  constexpr int ER = 64, EP = BN + 4;
  static_assert(J % 2 == 0 && ER * EP * 4 <= S * STAGE, "block columns in pairs, staging within the stages");
  __shared__ __attribute__((aligned(16))) uint8_t smem[S * STAGE + kScaleBytes<P, BM, BN, 4>];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave >> 1, wn = wave & 1;
  const TilePlace at = place(tiles_m, tiles_n, BM, BNO);
  uint32_t oa[CHA], ob[CHB];
#pragma unroll
  for (int c = 0; c < CHA; ++c) {
    const int row = 8 * (wave + NW * c) + (lane >> 3);
    oa[c] = uint32_t(min(int64_t(row), g.m - 1 - at.m0) * g.lda) + ((lane & 7) ^ row_swizzle(row)) * 16;
  }
#pragma unroll
  for (int c = 0; c < CHB; ++c) {
    const int row = 8 * (wave + NW * c) + (lane >> 3);
    ob[c] = uint32_t(min(int64_t(b_row<GATED>(row)), g.n - 1 - at.n0) * g.ldb) + ((lane & 7) ^ row_swizzle(row)) * 16;
  }
  v4f acc[I][J];
  ring_k_loop<FA, FB, BM, BN, S>(uniform(g.a + at.m0 * g.lda), b_base<GATED>(g, at.n0), oa, ob, int(g.k), smem, acc,
                                 tile_scales<BM, BN, 4>(g, at, S * STAGE));

  float *ep = reinterpret_cast<float *>(smem);
  const int fr = lane & 15, fq = lane >> 4;
  const SumScale s0 = scale_of(g, g.b_scale_inv), s1 = GATED ? scale_of(g, g.b2_scale_inv) : s0;
  constexpr int RW = ER < TM ? ER : TM;  // rows a wave stages per pass
#pragma unroll
  for (int p = 0; p < BM / ER; ++p) {
    __syncthreads();  // the last reads of the stages (or of the previous pass) are done
    if (TM < ER || wm == p * ER / TM) {
#pragma unroll
      for (int i = 0; i < RW / 16; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const v4f a = acc[TM < ER ? i : (p * ER % TM) / 16 + i][j];
          *reinterpret_cast<v4f *>(ep + ((TM < ER ? wm * TM : 0) + i * 16 + fr) * EP + wn * TN + j * 16 + 4 * fq) =
              scaled(a, j % 2 == 0 ? s0 : s1);
        }
    }
    __syncthreads();
    finish_rows<GATED, ER, BNO, 256, EP>(g, ep, tid, at.m0 + p * ER, at.n0);
  }
}

// Up to 16 rows (a token or a few being served): every operand row of B is read once
// and by one workgroup, so the product is bound by streaming B from memory, and
// what a tile kernel does for reuse (LDS stages, barriers) only costs latency.
// (Also for more rows where few_blocks says so.)
// A workgroup takes 16 rows and 16 OB outputs; its W waves split the reduction, K tile t to
// wave t % W.  A wave loads its fragments straight into registers, U K tiles
// in flight (lane l: row l % 16, bytes 16 (l / 16) of either half of the 128,
// the same for both operands), and the waves' sums meet in LDS, added in order.
// With a scale for each block the waves take four neighbouring K tiles at a time,
// whose scales are one word of a row.
template <bool GATED, int FA, int FB, int OB, int W, typename P>
__device__ __forceinline__ void act_rows_tile(const P &g, int blocks_n) {
  constexpr int NB = GATED ? 2 * OB : OB;  // 16-row blocks of B
  constexpr int U = 4;                     // K tiles in flight
  constexpr int EP = 16 * NB + 4;
  __shared__ __attribute__((aligned(16))) float sums[W][16 * EP];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  const int fr = lane & 15, fq = lane >> 4;
  const int64_t m0 = int64_t(int(blockIdx.x) / blocks_n) * 16, n0 = int64_t(int(blockIdx.x) % blocks_n) * (16 * OB);
  const int T = int((g.k + BK - 1) / BK), ktail = int(g.k % BK);

  const uint8_t *pa = g.a + min(m0 + fr, g.m - 1) * g.lda, *pb[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) {  // gated: gates and ups in alternating blocks
    const int64_t row = min(n0 + 16 * (GATED ? j / 2 : j) + fr, g.n - 1);
    pb[j] = (GATED && j % 2 == 1 ? g.b2 : g.b) + row * g.ldb;
  }
  v4f acc[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) acc[j] = v4f{0.f, 0.f, 0.f, 0.f};

  // The lane's 32 bytes of K tile t.
  auto load = [&](const uint8_t *p, int t) -> v8i {
    int c0 = fq, c1 = 4 + fq;
    if (ktail != 0 && t == T - 1) {  // chunks past the row's last 16 bytes re-read it; masked below
      const int last = (ktail - 1) >> 4;
      c0 = min(c0, last);
      c1 = min(c1, last);
    }
    const uint4 lo = *reinterpret_cast<const uint4 *>(p + int64_t(t) * BK + 16 * c0);
    const uint4 hi = *reinterpret_cast<const uint4 *>(p + int64_t(t) * BK + 16 * c1);
    return v8i{int(lo.x), int(lo.y), int(lo.z), int(lo.w), int(hi.x), int(hi.y), int(hi.z), int(hi.w)};
  };
  auto masked = [&](v8i f) -> v8i {
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const int nb = ktail - (q < 4 ? 16 * fq : 64 + 16 * fq) - 4 * (q % 4);  // bytes of this word to keep
      f[q] &= int(uint32_t((uint64_t(1) << (8 * (nb <= 0 ? 0 : (nb >= 4 ? 4 : nb)))) - 1u));
    }
    return f;
  };
  constexpr bool SC = kBlocked<P>;
  const uint8_t *ea = nullptr, *eb[NB];
  if constexpr (SC) {
    ea = g.a_exps + (min(m0 + fr, g.m - 1) >> g.a_shift) * g.ld_a_exps;
#pragma unroll
    for (int j = 0; j < NB; ++j) eb[j] = g.b_exps + (min(n0 + 16 * j + fr, g.n - 1) >> g.b_shift) * g.ld_b_exps;
  }
  constexpr int TS = SC ? 1 : W;  // K tiles between the U that a wave has in flight
  for (int t0 = SC ? U * wave : wave; t0 < T; t0 += U * W) {
    v8i fa[U], fb[U][NB];
    uint32_t sa = 0, sb[NB];
    if constexpr (SC) {
      sa = *reinterpret_cast<const uint32_t *>(ea + t0);
#pragma unroll
      for (int j = 0; j < NB; ++j) sb[j] = *reinterpret_cast<const uint32_t *>(eb[j] + t0);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = min(t0 + u * TS, T - 1);  // past the end: the last tile again, not used
#pragma unroll
      for (int j = 0; j < NB; ++j) fb[u][j] = load(pb[j], t);
      fa[u] = load(pa, t);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t0 + u * TS;
      if (t >= T) break;
      if (ktail != 0 && t == T - 1) {
#pragma unroll
        for (int j = 0; j < NB; ++j) fb[u][j] = masked(fb[u][j]);
        fa[u] = masked(fa[u]);
      }
#pragma unroll
      for (int j = 0; j < NB; ++j)
        if constexpr (SC)
          acc[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[u][j], fa[u], acc[j], FB, FA, 0, int(sb[j] >> (8 * u)), 0,
                                                                    int(sa >> (8 * u)));
        else
          acc[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[u][j], fa[u], acc[j], FB, FA, 0, 0, 0, 0);
    }
  }
  const SumScale s0 = scale_of(g, g.b_scale_inv), s1 = GATED ? scale_of(g, g.b2_scale_inv) : s0;
#pragma unroll
  for (int j = 0; j < NB; ++j) *reinterpret_cast<v4f *>(sums[wave] + fr * EP + 16 * j + 4 * fq) = acc[j];
  __syncthreads();
  // sums of the waves, scaled, into the first one's place
  for (int q = threadIdx.x; q < 16 * 4 * NB; q += 64 * W) {
    const int row = q / (4 * NB), col = q % (4 * NB) * 4;
    v4f s = *reinterpret_cast<const v4f *>(sums[0] + row * EP + col);
#pragma unroll
    for (int w = 1; w < W; ++w) s += *reinterpret_cast<const v4f *>(sums[w] + row * EP + col);
    const bool second = (col / 16) % 2 != 0;
    *reinterpret_cast<v4f *>(sums[0] + row * EP + col) = scaled(s, SumScale{second ? s1.a : s0.a, second ? s1.b : s0.b});
  }
  __syncthreads();
  if (threadIdx.x < 64) finish_rows<GATED, 16, 16 * OB, 64, EP>(g, sums[0], lane, m0, n0);
}

}  // namespace
}  // namespace qe
