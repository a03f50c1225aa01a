// FP8 encoding and the transposing LDS tile, shared by the kernels that write a
// tensor's codes both row-wise and transposed (quantize.hip, act_grad.hip).
#pragma once

#include "bf16.h"
#include "kernels.h"

namespace qe {
namespace {

constexpr int kTile = 128;
constexpr int kThreads = 256;

// Vectors at element (input) and byte (code) alignment.
typedef unsigned int u32x4_in __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned int u32x4_out __attribute__((ext_vector_type(4), aligned(1)));
typedef unsigned int u32x2_out __attribute__((ext_vector_type(2), aligned(1)));
typedef unsigned int u32_out __attribute__((aligned(1)));

// Four scaled values -> four FP8 codes, byte i = value i.  The hardware
// conversion rounds to nearest even but neither saturates (it overflows to
// NaN / inf) nor keeps the sign of a NaN, so values are clamped first with
// med3, which maps NaN to -fmax; NaN inputs are repaired separately.
template <int FMT>
__device__ __forceinline__ uint32_t enc4(float a, float b, float c, float d) {
  constexpr float fm = FMT == 0 ? 448.0f : 57344.0f;
  const float ca = __builtin_amdgcn_fmed3f(a, -fm, fm);
  const float cb = __builtin_amdgcn_fmed3f(b, -fm, fm);
  const float cc = __builtin_amdgcn_fmed3f(c, -fm, fm);
  const float cd = __builtin_amdgcn_fmed3f(d, -fm, fm);
  int r;
  if constexpr (FMT == 0) {
    r = __builtin_amdgcn_cvt_pk_fp8_f32(ca, cb, 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(cc, cd, r, true);
  } else {
    r = __builtin_amdgcn_cvt_pk_bf8_f32(ca, cb, 0, false);
    r = __builtin_amdgcn_cvt_pk_bf8_f32(cc, cd, r, true);
  }
  return uint32_t(r);
}

// The same for values that are known to be within +-fmax.
template <int FMT>
__device__ __forceinline__ uint32_t enc4_in_range(float a, float b, float c, float d) {
  int r;
  if constexpr (FMT == 0) {
    r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
  } else {
    r = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, 0, false);
    r = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, r, true);
  }
  return uint32_t(r);
}

// NaN -> 0x7F with the input's sign bit, for the rare thread that saw one.
__device__ __forceinline__ uint32_t nan_fix(uint32_t u, int byte, float v) {
  if (v != v) {
    const uint32_t code = 0x7fu | ((__float_as_uint(v) >> 24) & 0x80u);
    u = (u & ~(0xffu << (8 * byte))) | (code << (8 * byte));
  }
  return u;
}

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// A lane of phase 2 reads RPL consecutive rows; the swizzle follows its block.
template <int RPL>
__device__ __forceinline__ uint32_t lds_chunk_offset(int row, int chunk) {
  return uint32_t(row) * kTile + (uint32_t((chunk ^ (row / RPL)) & 7) << 4);
}

__device__ __forceinline__ uint32_t byte_of(uint32_t w, int j) { return (w >> (8 * j)) & 0xffu; }

}  // namespace
}  // namespace qe
