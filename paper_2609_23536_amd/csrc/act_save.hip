// 8-bit activation checkpoints (gfx950): an activation to int8 codes with one
// exponent byte per 32 columns of a row (the format in act.h), and back.
//
// HBM-bound: a save reads 2 or 4 bytes per value and writes 33/32, a restore the
// other way round.  A workgroup takes 64 rows x 128 columns, a lane eight
// columns of every sixteenth row: a group is four neighbouring lanes, which
// share its maximum by lane permutes.
#include "act.h"

namespace qe {
namespace {

typedef float f32x4_in __attribute__((ext_vector_type(4), aligned(4)));
constexpr int kRows = 64;

template <bool BF16>
__global__ __launch_bounds__(kThreads) void act_save_kernel(SaveParams p, int64_t tiles_c) {
  const int tid = threadIdx.x;
  const int64_t r0 = int64_t(blockIdx.x) / tiles_c * kRows;
  const int64_t col = int64_t(blockIdx.x) % tiles_c * kTile + (tid & 15) * 8;
  const int nc = int(p.cols - col < 0 ? 0 : (p.cols - col > 8 ? 8 : p.cols - col));
#pragma unroll
  for (int st = 0; st < kRows / 16; ++st) {
    const int64_t row = r0 + st * 16 + (tid >> 4);
    const int nv = row < p.rows ? nc : 0;
    f32x4 a = {0.f, 0.f, 0.f, 0.f}, b = a;
    if constexpr (BF16) {
      const uint16_t *src = static_cast<const uint16_t *>(p.x) + row * p.ld + col;
      if (nv == 8) {
        const u32x4_in w = *reinterpret_cast<const u32x4_in *>(src);
        a = f32x4{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xffff0000u), __uint_as_float(w[1] << 16),
                  __uint_as_float(w[1] & 0xffff0000u)};
        b = f32x4{__uint_as_float(w[2] << 16), __uint_as_float(w[2] & 0xffff0000u), __uint_as_float(w[3] << 16),
                  __uint_as_float(w[3] & 0xffff0000u)};
      } else if (nv > 0) {  // single elements, the last one again past it: no load waits for another
        uint32_t x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = src[e < nv ? e : nv - 1];
#pragma unroll
        for (int e = 0; e < 8; ++e) (e < 4 ? a : b)[e % 4] = e < nv ? bf16_to_f32(x[e]) : 0.0f;
      }
    } else {
      const float *src = static_cast<const float *>(p.x) + row * p.ld + col;
      if (nv == 8) {
        a = *reinterpret_cast<const f32x4_in *>(src);
        b = *reinterpret_cast<const f32x4_in *>(src + 4);
      } else if (nv > 0) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = src[e < nv ? e : nv - 1];
#pragma unroll
        for (int e = 0; e < 8; ++e) (e < 4 ? a : b)[e % 4] = e < nv ? x[e] : 0.0f;
      }
    }
    const uint32_t byte = save_exponent(max_lanes4(nan_max(amax4(a), amax4(b))));
    const uint32_t w0 = save_codes(a, byte), w1 = save_codes(b, byte);
    uint8_t *dst = static_cast<uint8_t *>(p.saved.data) + row * p.saved.ld + col;
    if (nv == 8) {
      *reinterpret_cast<u32x2_out *>(dst) = u32x2_out{w0, w1};
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < nv) dst[e] = uint8_t(byte_of(e < 4 ? w0 : w1, e % 4));
    }
    if (nv > 0 && (col & (kSaveGroup - 1)) == 0) p.saved.exps[row * p.saved.ld_exps + col / kSaveGroup] = uint8_t(byte);
  }
}

template <bool BF16>
__global__ __launch_bounds__(kThreads) void act_restore_kernel(SaveParams p, int64_t tiles_c) {
  const int tid = threadIdx.x;
  const int64_t r0 = int64_t(blockIdx.x) / tiles_c * kRows;
  const int64_t col = int64_t(blockIdx.x) % tiles_c * kTile + (tid & 15) * 8;
  const int nc = int(p.cols - col < 0 ? 0 : (p.cols - col > 8 ? 8 : p.cols - col));
#pragma unroll
  for (int st = 0; st < kRows / 16; ++st) {
    const int64_t row = r0 + st * 16 + (tid >> 4);
    const int nv = row < p.rows ? nc : 0;
    if (nv == 0) continue;
    const uint8_t *src = static_cast<const uint8_t *>(p.saved.data) + row * p.saved.ld + col;
    u32x2_out w = {0u, 0u};
    if (nv == 8) {
      w = *reinterpret_cast<const u32x2_out *>(src);
    } else {
      uint32_t x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = src[e < nv ? e : nv - 1];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e / 4] |= (e < nv ? x[e] : 0u) << (8 * (e % 4));
    }
    const uint32_t byte = p.saved.exps[row * p.saved.ld_exps + col / kSaveGroup];
    const f32x4 a = restore4(w[0], byte), b = restore4(w[1], byte);
    if constexpr (BF16) {
      uint16_t *dst = static_cast<uint16_t *>(p.x) + row * p.ld + col;
      const u32x4_in v = {bf16x2_bits(a[0], a[1]), bf16x2_bits(a[2], a[3]), bf16x2_bits(b[0], b[1]), bf16x2_bits(b[2], b[3])};
      if (nv == 8) {
        *reinterpret_cast<u32x4_in *>(dst) = v;
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < nv) dst[e] = uint16_t(v[e / 2] >> (16 * (e % 2)));
      }
    } else {
      float *dst = static_cast<float *>(p.x) + row * p.ld + col;
      if (nv == 8) {
        *reinterpret_cast<f32x4_in *>(dst) = a;
        *reinterpret_cast<f32x4_in *>(dst + 4) = b;
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < nv) dst[e] = (e < 4 ? a : b)[e % 4];
      }
    }
  }
}

template <typename K>
hipError_t launch_tiles(K bf16, K f32, const SaveParams &p, hipStream_t s) {
  if (p.rows <= 0 || p.cols <= 0) return hipSuccess;
  const int64_t tiles_c = (p.cols + kTile - 1) / kTile, tiles = (p.rows + kRows - 1) / kRows * tiles_c;
  if (tiles >= int64_t(1) << 31) return hipErrorInvalidValue;
  return klaunch(p.x_bf16 ? bf16 : f32, dim3(unsigned(tiles)), dim3(kThreads), 0, s, p, tiles_c);
}

}  // namespace

hipError_t launch_act_save(const SaveParams &p, hipStream_t s) {
  return launch_tiles(act_save_kernel<true>, act_save_kernel<false>, p, s);
}
hipError_t launch_act_restore(const SaveParams &p, hipStream_t s) {
  return launch_tiles(act_restore_kernel<true>, act_restore_kernel<false>, p, s);
}

}  // namespace qe
