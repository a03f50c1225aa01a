// FP8 codes with a power-of-two scale for each block of 128 values: the exponent
// byte of a block, codes at it, and rows of FP32 or BF16 values eight at a time
// (block_cast.hip, residual_norm.hip).
//
// Of a block with a = max |x|, e = floor(log2(fmax / a)) clamped to [-126, 126]
// (126 for a = 0), code = x 2^e rounded to nearest even, byte = 127 - e.  With
// a = m 2^E and fmax = 1.75 * 2^Emax the byte is a's exponent field less Emax, one
// more where m > 1.75: the carry of the addition below.  |x| 2^e <= fmax, so codes
// need no clamp.  A block that holds an infinity or a NaN gets the byte 255 (which
// the matrix instruction takes for NaN too) and NaN codes throughout.
#pragma once

#include "act.h"

namespace qe {
namespace {

constexpr int kBlock = 128;

template <int FMT>
__device__ __forceinline__ uint32_t block_byte(float amax) {
  const uint32_t a = abs_bits(amax);
  const int b = int((a + 0x1fffffu) >> 23) - (FMT == 0 ? 8 : 15);
  return a >= 0x7f800000u ? 255u : uint32_t(b < 1 ? 1 : b);
}
typedef short i16x2 __attribute__((ext_vector_type(2)));
// A block's scale as the conversions take it, 2^(byte - 127) (infinity for 255: they then give NaN).
__device__ __forceinline__ float block_step(uint32_t byte) { return __uint_as_float(byte << 23); }

// Two values at a block's scale -> two codes in the lower or upper half of `w`.  The
// instructions divide by the scale and round to nearest even; over all BF16 values (and
// FP32 ones with other low bits) and scales from 2^-126 to 2^126 their codes are those of
// x 2^e converted without a scale, checked on MI355X.
template <int FMT, bool HI>
__device__ __forceinline__ uint32_t convert_bf16(uint32_t w, uint32_t pair, float step) {
  const i16x2 old = __builtin_bit_cast(i16x2, w);
  const bf16x2_t x = __builtin_bit_cast(bf16x2_t, pair);
  return __builtin_bit_cast(uint32_t, FMT == 0 ? __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(old, x, step, HI)
                                               : __builtin_amdgcn_cvt_scalef32_pk_bf8_bf16(old, x, step, HI));
}
template <int FMT, bool HI>
__device__ __forceinline__ uint32_t convert_f32(uint32_t w, float a, float b, float step) {
  const i16x2 old = __builtin_bit_cast(i16x2, w);
  return __builtin_bit_cast(uint32_t, FMT == 0 ? __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(old, a, b, step, HI)
                                               : __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(old, a, b, step, HI));
}

// Four values -> four codes.
template <int FMT>
__device__ __forceinline__ uint32_t block_codes(const float *x, float step) {
  return convert_f32<FMT, true>(convert_f32<FMT, false>(0u, x[0], x[1], step), x[2], x[3], step);
}

// Maximum over the 16 lanes of an aligned group, in all of them.
__device__ __forceinline__ float max_lanes16(float v) { return max_dpp<0x140>(max_lanes8(v)); }  // 15 - lane
typedef float f32x4_in __attribute__((ext_vector_type(4), aligned(4)));

// Row `row` of a matrix: uniform in a workgroup where `row` is, so that a lane's
// address is a scalar base and its column's 32-bit offset.
__device__ __forceinline__ char *row_of(const MatrixRef &m, bool bf16, int64_t row) {
  return static_cast<char *>(m.data) + row * m.ld * (bf16 ? 2 : 4);
}

// Eight consecutive values from column `at` of a row, n of which exist (the others are zero).
__device__ __forceinline__ void load8(const void *base, bool bf16, uint32_t at, int n, float *f) {
  if (bf16) {
    const uint16_t *p = static_cast<const uint16_t *>(base) + at;
    if (n >= 8) {
      const u32x4_in w = *reinterpret_cast<const u32x4_in *>(p);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f[2 * e] = __uint_as_float(w[e] << 16);
        f[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = e < n ? bf16_to_f32(p[e]) : 0.0f;
    }
  } else {
    const float *p = static_cast<const float *>(base) + at;
    if (n >= 8) {
      const f32x4_in a = *reinterpret_cast<const f32x4_in *>(p), b = *reinterpret_cast<const f32x4_in *>(p + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f[e] = a[e];
        f[4 + e] = b[e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = e < n ? p[e] : 0.0f;
    }
  }
}

__device__ __forceinline__ void store8(void *base, bool bf16, uint32_t at, int n, const float *f) {
  if (bf16) {
    uint16_t *p = static_cast<uint16_t *>(base) + at;
    if (n >= 8) {
      *reinterpret_cast<u32x4_in *>(p) = u32x4_in{bf16x2_bits(f[0], f[1]), bf16x2_bits(f[2], f[3]), bf16x2_bits(f[4], f[5]),
                                                  bf16x2_bits(f[6], f[7])};
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < n) p[e] = bf16_bits(f[e]);
    }
  } else {
    float *p = static_cast<float *>(base) + at;
    if (n >= 8) {
      *reinterpret_cast<f32x4_in *>(p) = f32x4_in{f[0], f[1], f[2], f[3]};
      *reinterpret_cast<f32x4_in *>(p + 4) = f32x4_in{f[4], f[5], f[6], f[7]};
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < n) p[e] = f[e];
    }
  }
}

// Codes that leave in whole lines of 128 bytes go past the caches, and what is read stays
// there; codes that share lines do not.  MI355X, us, cached / past them: cast of BF16 4096 x
// 4096 18.5 / 18.2, its input in the caches 12.6 / 9.4; 4096 x 14336 54.2 / 51.6; 8192 x
// 8192 70.0 / 66.2; with 4000 x 14000, where lines are shared, 71 / 89.
inline bool whole_lines(const BlockedRef &b) { return uintptr_t(b.data) % 128 == 0 && b.ld % 128 == 0; }

template <typename V>
__device__ __forceinline__ void store_out(uint8_t *p, V v, bool past) {
  // (the empty statements keep the compiler from making one ordinary store of the two)
  if (past) {
    __builtin_nontemporal_store(v, reinterpret_cast<V *>(p));
    asm volatile("");
  } else {
    asm volatile("");
    *reinterpret_cast<V *>(p) = v;
  }
}

// Eight codes of a row, n of which exist.
__device__ __forceinline__ void store_codes8(uint8_t *p, int n, uint32_t lo, uint32_t hi, bool past) {
  if (n >= 8) {
    store_out(p, u32x2_out{lo, hi}, past);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = uint8_t(byte_of(e < 4 ? lo : hi, e % 4));
  }
}

}  // namespace
}  // namespace qe
