// Activations, their slopes and the 8-bit checkpoint format, as device
// functions of the kernels that read or write them (act_gemm.hip,
// act_grad.hip, act_save.hip).
#pragma once

#include "fp8_enc.h"

namespace qe {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------- activations
// With p(t) = 1 / (1 + e^-t):
//   silu(z) = z p(z)                       silu'(z) = p (1 + z (1 - p))
//   gelu(z) = z Phi(z)                     gelu'(z) = Phi + z phi(z)
//   gelu_tanh(z) = z p(2 c (z + b z^3))    since (1 + tanh t) / 2 = p(2 t),
//   gelu_tanh'(z) = P + z P (1 - P) 2 c (1 + 3 b z^2),  c = sqrt(2 / pi), b = 0.044715
// e^-t is the hardware's 2^x (1 ulp) of a once rounded product, and the
// quotient the hardware's reciprocal (1 ulp): a relative error of about
// (2 + |t|) 2^-24, far below the BF16 the values are usually rounded to.
__device__ __forceinline__ float sigmoid(float t) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(t * -1.44269504088896340736f));
}
constexpr float kGelu2C = 1.59576912160573071176f;  // 2 sqrt(2 / pi)
constexpr float kGeluB = 0.044715f;
constexpr float kGeluFar = 256.0f;  // z^2 from which P is 0 or 1 in 32 bits; keeps z P (1 - P) z^2 off 0 * inf

// Phi(z) and e = exp(-z^2 / 2), without a branch.  |z| < 1.5: Taylor's series of
// Phi(z) - 1/2 to z^21 (the next term is below 2.4e-9; with coefficients of FP32 the
// sum is off by 1.0e-8).  Beyond, on the negative side, where nothing may cancel:
// Phi(-a) = t P(t) e with t = 1 / (1 + 0.45 a), P of degree 6 fitted to Phi(-a) / (t e)
// over a >= 1.5, relative error below 2.6e-7 there.  With its roundings off by at
// most 7.1e-8 over z in -9 .. 9, as erf in FP32 is (6.1e-8; the shorter form of
// Abramowitz and Stegun 7.1.26, off by 7.5e-8 before rounding, moved ten times as
// many FP8 codes of a gradient as erf did).
__device__ __forceinline__ float normal_cdf(float z, float &e) {
  const float q = z * z, a = __builtin_fabsf(z);
  float c = 5.112434781e-12f;
  c = __builtin_fmaf(c, q, -1.1301171804e-10f);
  c = __builtin_fmaf(c, q, 2.2735298088e-09f);
  c = __builtin_fmaf(c, q, -4.1226673630e-08f);
  c = __builtin_fmaf(c, q, 6.6596936676e-07f);
  c = __builtin_fmaf(c, q, -9.4446559160e-06f);
  c = __builtin_fmaf(c, q, 1.1543469009e-04f);
  c = __builtin_fmaf(c, q, -1.1873282492e-03f);
  c = __builtin_fmaf(c, q, 9.9735567346e-03f);
  c = __builtin_fmaf(c, q, -6.6490381956e-02f);
  c = __builtin_fmaf(c, q, 3.9894229174e-01f);
  const float near = __builtin_fmaf(z, c, 0.5f);
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(a, 0.45f, 1.0f));
  e = __builtin_amdgcn_exp2f(q * -0.72134752044448170368f);
  float s = 0.09566925466060638f;
  s = __builtin_fmaf(s, t, -0.17652954161167145f);
  s = __builtin_fmaf(s, t, 0.015372074209153652f);
  s = __builtin_fmaf(s, t, 0.06544602662324905f);
  s = __builtin_fmaf(s, t, 0.14354704320430756f);
  s = __builtin_fmaf(s, t, 0.17951330542564392f);
  s = __builtin_fmaf(s, t, 0.17952407896518707f);
  s *= t * e;  // Phi(-a)
  return a < 1.5f ? near : (z < 0.0f ? s : 1.0f - s);
}

template <int ACT>
__device__ __forceinline__ float act_value(float z) {
  if constexpr (ACT == kActRelu) return z < 0.0f ? 0.0f : z;  // NaN stays
  if constexpr (ACT == kActGelu) {
    float e;
    return z * normal_cdf(z, e);
  }
  if constexpr (ACT == kActGeluTanh) return z * sigmoid(kGelu2C * z * (1.0f + kGeluB * fminf(z * z, kGeluFar)));
  if constexpr (ACT == kActSilu) return z * sigmoid(z);
  return z;
}

// value and slope
template <int ACT>
__device__ __forceinline__ void act_both(float z, float &v, float &d) {
  if constexpr (ACT == kActRelu) {
    v = z < 0.0f ? 0.0f : z;
    d = z > 0.0f ? 1.0f : 0.0f;
  } else if constexpr (ACT == kActGelu) {
    float e;
    const float cdf = normal_cdf(z, e);
    v = z * cdf;
    d = cdf + z * (0.39894228040143267794f * e);
  } else if constexpr (ACT == kActGeluTanh) {
    const float q = fminf(z * z, kGeluFar);
    const float p = sigmoid(kGelu2C * z * (1.0f + kGeluB * q));
    v = z * p;
    d = p + v * (1.0f - p) * (kGelu2C * (1.0f + 3.0f * kGeluB * q));
  } else if constexpr (ACT == kActSilu) {
    const float p = sigmoid(z);
    v = z * p;
    d = p + v * (1.0f - p);
  } else {
    v = z;
    d = 1.0f;
  }
}

// Calls f.operator()<ACT>() for the (uniform) activation `act`.
template <typename F>
__device__ __forceinline__ void act_switch(int act, F &&f) {
  switch (act) {
    case kActRelu: f(std::integral_constant<int, kActRelu>{}); break;
    case kActGelu: f(std::integral_constant<int, kActGelu>{}); break;
    case kActGeluTanh: f(std::integral_constant<int, kActGeluTanh>{}); break;
    case kActSilu: f(std::integral_constant<int, kActSilu>{}); break;
    default: f(std::integral_constant<int, kActNone>{}); break;
  }
}

// ----------------------------------------------------------- 8-bit checkpoint
// 32 columns of a row share a step 2^-s, s = floor(log2(127 / amax)) clamped to
// [-126, 126]; a value is the int8 code rne(x 2^s), so |code| <= 127 and the
// error is at most half a step, amax / 127 at most (less than a step from 63.5 *
// 2^122 on, see save_codes).  The group's byte is
// 127 - s, the step's exponent field: amax's own exponent field less 6, one
// more where its mantissa is above 127/64 (the carry of the addition below).
// An infinity or a NaN makes the byte 255, whose step is infinite, with codes of
// zero: code * step is then NaN for the whole group.
// Steps that are powers of two keep the restored values exact in BF16 and FP32
// (a code has seven bits), scaling exact, and the byte count at 33/32.
constexpr int kSaveGroup = 32;

__device__ __forceinline__ uint32_t save_exponent(float group_max) {
  const uint32_t amax = abs_bits(group_max);
  const int e = int((amax + 0x1ffffu) >> 23) - 6;
  return amax >= 0x7f800000u ? 255u : uint32_t(e < 1 ? 1 : e);
}

// Four values -> four int8 codes.  x 2^s is exact; adding 1.5 * 2^23 rounds it
// to nearest even and leaves the code in the sum's low byte.  RARE: the byte
// may be the largest step's, 2^122, whose codes stop at 63 because 64 steps are
// 2^128, or 255.  Whether it may is asked once for all that a wave stores
// together: a branch around every four values cost 4% of a gated training pass.
constexpr uint32_t kSaveTopByte = 249u;
__device__ __forceinline__ bool save_rare(uint32_t byte) { return __builtin_amdgcn_ballot_w64(byte >= kSaveTopByte) != 0; }
template <bool RARE>
__device__ __forceinline__ uint32_t save_codes(f32x4 x, uint32_t byte) {
  if constexpr (RARE) {
    const float top = byte == kSaveTopByte ? 0x1.f8p127f : __builtin_inff();  // 63 steps
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = __builtin_amdgcn_fmed3f(x[e], -top, top);
  }
  const float mult = __uint_as_float((254u - byte) << 23);  // 2^s
  constexpr float kRound = 12582912.0f;
  const uint32_t b0 = __float_as_uint(__builtin_fmaf(x[0], mult, kRound)), b1 = __float_as_uint(__builtin_fmaf(x[1], mult, kRound));
  const uint32_t b2 = __float_as_uint(__builtin_fmaf(x[2], mult, kRound)), b3 = __float_as_uint(__builtin_fmaf(x[3], mult, kRound));
  const uint32_t lo = __builtin_amdgcn_perm(b1, b0, 0x0c0c0400u), hi = __builtin_amdgcn_perm(b3, b2, 0x04000c0cu);
  return RARE && byte == 255u ? 0u : lo | hi;
}

// Code j of a word, restored: a signed byte has a hardware conversion, and the
// product with the step is exact.  (Not as code + 128 with an addend of -128
// steps: that addend overflows for the steps 2^121 and 2^122 of large groups.)
template <int J>
__device__ __forceinline__ float restore_code(uint32_t word, float step) {
  return float(int8_t(word >> (8 * J))) * step;
}
__device__ __forceinline__ f32x4 restore4(uint32_t codes, uint32_t byte) {
  const float step = __uint_as_float(byte << 23);
  return f32x4{restore_code<0>(codes, step), restore_code<1>(codes, step), restore_code<2>(codes, step), restore_code<3>(codes, step)};
}

// Maxima that keep a NaN (one instruction for three operands on gfx950).
__device__ __forceinline__ float nan_max(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float amax4(f32x4 x) {
  return nan_max(nan_max(__builtin_fabsf(x[0]), __builtin_fabsf(x[1])), nan_max(__builtin_fabsf(x[2]), __builtin_fabsf(x[3])));
}

// Maximum over the 4 (8) lanes of an aligned group of lanes, in all of them.
template <int CTRL>
__device__ __forceinline__ float max_dpp(float v) {
  return nan_max(v, __uint_as_float(uint32_t(__builtin_amdgcn_mov_dpp(int(__float_as_uint(v)), CTRL, 0xf, 0xf, true))));
}
__device__ __forceinline__ float max_lanes4(float v) { return max_dpp<0x4e>(max_dpp<0xb1>(v)); }  // lane ^ 1, lane ^ 2
__device__ __forceinline__ float max_lanes8(float v) { return max_dpp<0x141>(max_lanes4(v)); }     // 7 - lane within eight

// The same over lanes l, l ^ 16, l ^ 32 and l ^ 48: each exchange leaves one half's
// values in the first result and the other half's in the second, in all lanes.
__device__ __forceinline__ float max_lanes_by16(float v) {
  uint32_t b = __float_as_uint(v);
  auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
  b = __float_as_uint(nan_max(__uint_as_float(r[0]), __uint_as_float(r[1])));
  r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return nan_max(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

}  // namespace
}  // namespace qe
