// BF16 conversions of the gfx950 kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace qe {
namespace {

// Two floats to two bf16 (round to nearest even, NaN stays a quiet NaN with
// its sign and top payload bits) with the gfx950 packed conversion; bit-equal
// to the integer form (u + 0x7fff + ((u >> 16) & 1)) >> 16 on every input,
// which was checked on MI355X over all exponents, boundaries, denormals and NaNs.
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t bf16x2_bits(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{lo, hi}, bf16x2_t));
}
__device__ __forceinline__ uint16_t bf16_bits(float f) { return uint16_t(bf16x2_bits(f, 0.0f)); }
__device__ __forceinline__ float bf16_to_f32(uint32_t bits16) { return __uint_as_float(bits16 << 16); }

}  // namespace
}  // namespace qe
