// 8-bit activation checkpoints (gfx950): an activation to int8 codes with one
// exponent byte per 32 columns of a row (the format in act.h), and back.
//
// HBM-bound: a save reads 2 or 4 bytes per value and writes 33/32, a restore the
// other way round.  A workgroup takes 64 rows x 128 columns, a lane eight
// columns of every sixteenth row, all four loads in flight: a group is four
// neighbouring lanes, which share its maximum by lane permutes.  MI355X, BF16 4096 x
// 14336: saved in 36 us (5.0 TB/s) after the kernel that wrote it, in 42 from memory;
// restored in 29 (6.1).
//
// All accesses are ordinary: what is saved was written by the kernel before and
// is read again by the one after.  With non-temporal loads, MI355X, us from one to
// the other, ordinary / so: BF16 save 4096 x 14336 35.8 / 34.7, with the cast
// of the same tensor after it 74.1 / 79.9; 8192 x 28672 134 / 127 and 299 / 301; FP32
// 4096 x 14336 60.9 / 69.5 and 115 / 133.
#include "act.h"

namespace qe {
namespace {

typedef float f32x4_in __attribute__((ext_vector_type(4), aligned(4)));
constexpr int kRows = 64, kSteps = kRows / 16;

struct Eight {
  f32x4 a, b;
};

// Eight values of a row at `at`, of which nv exist (all, if FULL; the others
// read as zero).  Where some do not exist the last one is read again in their
// place, so that no load waits for another.
template <bool BF16, bool FULL>
__device__ __forceinline__ Eight load8(const void *base, int64_t at, int nv) {
  Eight r = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
  if constexpr (BF16) {
    const uint16_t *p = static_cast<const uint16_t *>(base) + at;
    if (FULL || nv == 8) {
      const u32x4_in w = *reinterpret_cast<const u32x4_in *>(p);
      r.a = f32x4{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xffff0000u), __uint_as_float(w[1] << 16),
                  __uint_as_float(w[1] & 0xffff0000u)};
      r.b = f32x4{__uint_as_float(w[2] << 16), __uint_as_float(w[2] & 0xffff0000u), __uint_as_float(w[3] << 16),
                  __uint_as_float(w[3] & 0xffff0000u)};
    } else if (nv > 0) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = bf16_to_f32(p[e < nv ? e : nv - 1]);
#pragma unroll
      for (int e = 0; e < 8; ++e) (e < 4 ? r.a : r.b)[e % 4] = e < nv ? x[e] : 0.0f;
    }
  } else {
    const float *p = static_cast<const float *>(base) + at;
    if (FULL || nv == 8) {
      r.a = *reinterpret_cast<const f32x4_in *>(p);
      r.b = *reinterpret_cast<const f32x4_in *>(p + 4);
    } else if (nv > 0) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = p[e < nv ? e : nv - 1];
#pragma unroll
      for (int e = 0; e < 8; ++e) (e < 4 ? r.a : r.b)[e % 4] = e < nv ? x[e] : 0.0f;
    }
  }
  return r;
}

template <bool BF16, bool FULL>
__device__ __forceinline__ void save_tile(const SaveParams &p, int64_t row0, int64_t col) {
  const int nc = FULL ? 8 : int(p.cols - col < 0 ? 0 : (p.cols - col > 8 ? 8 : p.cols - col));
  Eight x[kSteps];
#pragma unroll
  for (int st = 0; st < kSteps; ++st)
    x[st] = load8<BF16, FULL>(p.x, (row0 + st * 16) * p.ld + col, FULL || row0 + st * 16 < p.rows ? nc : 0);
  uint32_t byte[kSteps], most = 0u;
#pragma unroll
  for (int st = 0; st < kSteps; ++st) {
    byte[st] = save_exponent(max_lanes4(nan_max(amax4(x[st].a), amax4(x[st].b))));
    most = byte[st] > most ? byte[st] : most;
  }
  auto store = [&](auto rare) {
    constexpr bool RARE = decltype(rare)::value;
#pragma unroll
    for (int st = 0; st < kSteps; ++st) {
      const int64_t row = row0 + st * 16;
      const int nv = FULL || row < p.rows ? nc : 0;
      const uint32_t w0 = save_codes<RARE>(x[st].a, byte[st]), w1 = save_codes<RARE>(x[st].b, byte[st]);
      uint8_t *dst = static_cast<uint8_t *>(p.saved.data) + row * p.saved.ld + col;
      if (FULL || nv == 8) {
        *reinterpret_cast<u32x2_out *>(dst) = u32x2_out{w0, w1};
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < nv) dst[e] = uint8_t(byte_of(e < 4 ? w0 : w1, e % 4));
      }
      if (nv > 0 && (col & (kSaveGroup - 1)) == 0) p.saved.exps[row * p.saved.ld_exps + col / kSaveGroup] = uint8_t(byte[st]);
    }
  };
  if (__builtin_expect(save_rare(most), 0))
    store(std::true_type{});
  else
    store(std::false_type{});
}

template <bool BF16, bool FULL>
__device__ __forceinline__ void restore_tile(const SaveParams &p, int64_t row0, int64_t col) {
  const int nc = FULL ? 8 : int(p.cols - col < 0 ? 0 : (p.cols - col > 8 ? 8 : p.cols - col));
  u32x2_out w[kSteps];
  uint32_t byte[kSteps];
#pragma unroll
  for (int st = 0; st < kSteps; ++st) {
    const int64_t row = row0 + st * 16;
    const int nv = FULL || row < p.rows ? nc : 0;
    w[st] = u32x2_out{0u, 0u};
    byte[st] = 0u;
    if (nv == 0) continue;
    const uint8_t *src = static_cast<const uint8_t *>(p.saved.data) + row * p.saved.ld + col;
    if (FULL || nv == 8) {
      w[st] = *reinterpret_cast<const u32x2_out *>(src);
    } else {
      uint32_t x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = src[e < nv ? e : nv - 1];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[st][e / 4] |= (e < nv ? x[e] : 0u) << (8 * (e % 4));
    }
    byte[st] = p.saved.exps[row * p.saved.ld_exps + col / kSaveGroup];
  }
#pragma unroll
  for (int st = 0; st < kSteps; ++st) {
    const int64_t row = row0 + st * 16;
    const int nv = FULL || row < p.rows ? nc : 0;
    const f32x4 a = restore4(w[st][0], byte[st]), b = restore4(w[st][1], byte[st]);
    if constexpr (BF16) {
      uint16_t *dst = static_cast<uint16_t *>(p.x) + row * p.ld + col;
      const u32x4_in v = {bf16x2_bits(a[0], a[1]), bf16x2_bits(a[2], a[3]), bf16x2_bits(b[0], b[1]), bf16x2_bits(b[2], b[3])};
      if (FULL || nv == 8) {
        *reinterpret_cast<u32x4_in *>(dst) = v;
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < nv) dst[e] = uint16_t(v[e / 2] >> (16 * (e % 2)));
      }
    } else {
      float *dst = static_cast<float *>(p.x) + row * p.ld + col;
      if (FULL || nv == 8) {
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

template <bool SAVE, bool BF16>
__global__ __launch_bounds__(kThreads) void act_checkpoint_kernel(SaveParams p, int64_t tiles_c) {
  const int64_t r0 = int64_t(blockIdx.x) / tiles_c * kRows, c0 = int64_t(blockIdx.x) % tiles_c * kTile;
  const int64_t row = r0 + (threadIdx.x >> 4), col = c0 + (threadIdx.x & 15) * 8;
  const bool full = r0 + kRows <= p.rows && c0 + kTile <= p.cols;
  if constexpr (SAVE) {
    if (full)
      save_tile<BF16, true>(p, row, col);
    else
      save_tile<BF16, false>(p, row, col);
  } else {
    if (full)
      restore_tile<BF16, true>(p, row, col);
    else
      restore_tile<BF16, false>(p, row, col);
  }
}

template <bool SAVE>
hipError_t launch_tiles(const SaveParams &p, hipStream_t s) {
  if (p.rows <= 0 || p.cols <= 0) return hipSuccess;
  const int64_t tiles_c = (p.cols + kTile - 1) / kTile, tiles = (p.rows + kRows - 1) / kRows * tiles_c;
  if (tiles >= int64_t(1) << 31) return hipErrorInvalidValue;
  const dim3 grid{unsigned(tiles)}, block(kThreads);
  return p.x_bf16 ? klaunch(act_checkpoint_kernel<SAVE, true>, grid, block, 0, s, p, tiles_c)
                  : klaunch(act_checkpoint_kernel<SAVE, false>, grid, block, 0, s, p, tiles_c);
}

}  // namespace

hipError_t launch_act_save(const SaveParams &p, hipStream_t s) { return launch_tiles<true>(p, s); }
hipError_t launch_act_restore(const SaveParams &p, hipStream_t s) { return launch_tiles<false>(p, s); }

}  // namespace qe
