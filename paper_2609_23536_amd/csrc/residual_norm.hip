// The sum of a residual stream and a block's output with the norms before and after
// it, and its gradient (gfx950).  With f(v) = 1 / sqrt(mean v^2 + eps) of a row v:
//     p = y f(y) (o + w_post)  (or y),   r = x_scale x + y_scale gate p,
//     h = r f(r) (o + w_pre)
// r is rounded to the type it is stored in before f(r) and h are computed from it: the
// backward pass, and the kernel that casts h again for dW, read that r.  Everything
// else is FP32.
//
// Backward, with n = r f(r), m = y f(y):
//     t = dr + f(r) (d - n mean(d n)),  d = dh (o + w_pre)
//     dx = x_scale t,   b = y_scale t (the gradient of gate p),   dw_pre = sum dh n
//     dy = f(y) (e - m mean(e m)),  e = b gate (o + w_post)  (or b gate)
// and with S = sum b m over the rows that share a row of gates:
//     dgate = S (o + w_post),   dw_post = sum over the gates' rows of S gate
// so one sum of columns serves both.
//
// Both are bound by memory.  Forward: one workgroup a row, which stays in registers
// between the two sums.  Backward: a workgroup takes up to 16 rows that share their
// gates, one after the other, and keeps the column sums in registers; they go to the
// workspace once per 16 rows, and a second kernel adds them in a fixed order.
#include "block_scale.h"

#include <algorithm>
#include <initializer_list>

namespace qe {
namespace {

constexpr int kLanes = 1024;  // most lanes for a row

template <int CTRL>
__device__ __forceinline__ float add_dpp(float v) {
  return v + __uint_as_float(uint32_t(__builtin_amdgcn_mov_dpp(int(__float_as_uint(v)), CTRL, 0xf, 0xf, true)));
}
// Sum over the wave, in all lanes: lanes l ^ 1, l ^ 2, 7 - l and 15 - l within 8 and 16, then l ^ 16 and l ^ 32.
__device__ __forceinline__ float wave_sum(float v) {
  v = add_dpp<0x140>(add_dpp<0x141>(add_dpp<0x4e>(add_dpp<0xb1>(v))));
  uint32_t b = __float_as_uint(v);
  auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
  b = __float_as_uint(__uint_as_float(r[0]) + __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Sum over the workgroup, in all lanes; `red`: one float per wave, which no sum before
// the last one has used (a lane may still be reading what that one left).
__device__ __forceinline__ float group_sum(float v, float *red) {
  v = wave_sum(v);
  const int waves = int(blockDim.x) >> 6;
  if (waves == 1) return v;
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
  for (int w = 1; w < waves; ++w) v += red[w];
  return v;
}

// offset + weight of eight columns (1 without weights)
__device__ __forceinline__ void weights8(const void *w, bool bf16, uint32_t col, int n, float offset, float *f) {
  if (w == nullptr) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = 1.0f;
    return;
  }
  load8(w, bf16, col, n, f);
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] += offset;
}

template <bool BF16>
__device__ __forceinline__ bool is_bf16(const MatrixRef &m) {
  return BF16 || m.bf16 != 0;
}

template <int NV, bool BF16>
__global__ __launch_bounds__(kLanes) void residual_norm_kernel(ResidualParams p) {
  __shared__ float red[2][16];
  const int tid = threadIdx.x;
  const int64_t row = p.row0 + blockIdx.x;
  const float inv_cols = 1.0f / float(p.cols);
  const MatrixRef gates{const_cast<void *>(p.gate), p.ld_gate, p.gate_bf16, 0};
  float r[NV][8];
  uint32_t col[NV];
  int n[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    col[v] = (uint32_t(v) * blockDim.x + tid) * 8;
    n[v] = max(0, min(8, int(p.cols) - int(col[v])));
  }
  float x[NV][8];
  if (p.x.data != nullptr) {
#pragma unroll
    for (int v = 0; v < NV; ++v) load8(row_of(p.x, is_bf16<BF16>(p.x), row), is_bf16<BF16>(p.x), col[v], n[v], x[v]);
  }
  if (p.y.data != nullptr) {
    float sum = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) load8(row_of(p.y, is_bf16<BF16>(p.y), row), is_bf16<BF16>(p.y), col[v], n[v], r[v]);
    float f = 1.0f;
    if (p.post_norm) {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(r[v][e], r[v][e], sum);
      f = 1.0f / __builtin_sqrtf(group_sum(sum, red[0]) * inv_cols + p.post_eps);
      if (tid == 0 && p.post_rstd != nullptr) p.post_rstd[row] = f;
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (p.post_norm) {
        float w[8];
        weights8(p.post_weight, p.weight_bf16 != 0, col[v], n[v], p.offset, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) r[v][e] = r[v][e] * f * w[e];
      }
      if (p.gate != nullptr) {
        float g[8];
        load8(row_of(gates, p.gate_bf16 != 0, row / p.gate_rows), p.gate_bf16 != 0, col[v], n[v], g);
#pragma unroll
        for (int e = 0; e < 8; ++e) r[v][e] *= g[e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) r[v][e] *= p.y_scale;
    }
    if (p.x.data != nullptr) {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) r[v][e] = __builtin_fmaf(p.x_scale, x[v][e], r[v][e]);
    }
  } else {
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) r[v][e] = p.x_scale * x[v][e];
  }
  if (p.r.data != nullptr) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      store8(row_of(p.r, is_bf16<BF16>(p.r), row), is_bf16<BF16>(p.r), col[v], n[v], r[v]);
      if (is_bf16<BF16>(p.r)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) r[v][e] = bf16_to_f32(bf16_bits(r[v][e]));
      }
    }
  }
  if (!p.pre_norm) return;
  float sum = 0.0f;
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(r[v][e], r[v][e], sum);
  const float f = 1.0f / __builtin_sqrtf(group_sum(sum, red[1]) * inv_cols + p.pre_eps);
  if (tid == 0 && p.pre_rstd != nullptr) p.pre_rstd[row] = f;
  if (p.h.data == nullptr && p.row.data == nullptr) return;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    float w[8], h[8];
    weights8(p.pre_weight, p.weight_bf16 != 0, col[v], n[v], p.offset, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = e < n[v] ? r[v][e] * f * w[e] : 0.0f;
    if (p.h.data != nullptr) store8(row_of(p.h, is_bf16<BF16>(p.h), row), is_bf16<BF16>(p.h), col[v], n[v], h);
    if (p.row.data != nullptr) {
      const float a = max_lanes16(nan_max(amax4(f32x4{h[0], h[1], h[2], h[3]}), amax4(f32x4{h[4], h[5], h[6], h[7]})));
      uint8_t *dst = p.row.data + row * p.row.ld + col[v];
      const uint32_t byte = p.row.fmt == 0 ? block_byte<0>(a) : block_byte<1>(a);
      const float mult = block_mult(byte);
      if (p.row.fmt == 0)
        store_codes8(dst, n[v], block_codes<0>(h, mult), block_codes<0>(h + 4, mult));
      else
        store_codes8(dst, n[v], block_codes<1>(h, mult), block_codes<1>(h + 4, mult));
      if ((tid & 15) == 0 && n[v] > 0) p.row.exps[row * p.row.ld_exps + col[v] / kBlock] = uint8_t(byte);
    }
  }
}

// Eight values of a row as they are stored, where that is BF16: four registers.
__device__ __forceinline__ u32x4_in fetch8(const void *base, uint32_t at, int n) {
  const uint16_t *p = static_cast<const uint16_t *>(base) + at;
  if (n >= 8) return *reinterpret_cast<const u32x4_in *>(p);
  u32x4_in w = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (e < n) w[e / 2] |= uint32_t(p[e]) << (16 * (e % 2));
  return w;
}

// A row of one of the gradient's inputs.  Where all matrices are BF16 (and a lane has one vector) it is fetched a
// row ahead, so that the next row is on its way during this one's sums.
template <int NV, bool BF16>
struct Row {
  static constexpr bool kAhead = BF16 && NV == 1;
  u32x4_in w[kAhead ? NV : 1];
  __device__ __forceinline__ void fetch(const MatrixRef &m, int64_t row, const uint32_t (&col)[NV], const int (&n)[NV]) {
    if constexpr (kAhead) {
      if (m.data == nullptr) return;
#pragma unroll
      for (int v = 0; v < NV; ++v) w[v] = fetch8(row_of(m, true, row), col[v], n[v]);
    }
  }
  __device__ __forceinline__ void get(const MatrixRef &m, int64_t row, uint32_t col, int n, int v, float *f) const {
    if constexpr (kAhead) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f[2 * e] = __uint_as_float(w[v][e] << 16);
        f[2 * e + 1] = __uint_as_float(w[v][e] & 0xffff0000u);
      }
    } else {
      load8(row_of(m, is_bf16<BF16>(m), row), is_bf16<BF16>(m), col, n, f);
    }
  }
};

// Column sums of a lane's eight columns: in registers with one vector a lane, in LDS
// (the lane's own 16-byte slots) with two, where 128 registers a lane do not hold them.
template <int NV>
struct ColumnSums {
  static constexpr bool kInLds = NV > 1;
  f32x4 reg[kInLds ? 1 : 2];
  f32x4 *lds;
  __device__ __forceinline__ void clear(f32x4 *mem) {
    lds = mem + threadIdx.x;
    if constexpr (kInLds) {
#pragma unroll
      for (int q = 0; q < 2 * NV; ++q) lds[q * kLanes] = f32x4{0.f, 0.f, 0.f, 0.f};
    } else {
      reg[0] = reg[1] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  __device__ __forceinline__ void add(int v, const float *a, const float *b) {  // += a b
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f32x4 s = kInLds ? lds[(2 * v + h) * kLanes] : reg[kInLds ? 0 : h];
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] = __builtin_fmaf(a[4 * h + e], b[4 * h + e], s[e]);
      if constexpr (kInLds)
        lds[(2 * v + h) * kLanes] = s;
      else
        reg[h] = s;
    }
  }
  __device__ __forceinline__ void store(float *row, int v, uint32_t col, int n) const {
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = kInLds ? lds[(2 * v + e / 4) * kLanes][e % 4] : reg[kInLds ? 0 : e / 4][e % 4];
    store8(row, false, col, n, f);
  }
};

// Chunks of up to kGradRows rows: `per_group` of them for each group of gate_rows rows.
template <int NV, bool BF16>
__global__ __launch_bounds__(kLanes) void residual_grad_kernel(ResidualGradParams p, int64_t per_group, int64_t chunks) {
  __shared__ __attribute__((aligned(16))) float reds[4][kLanes / 64];
  const int tid = threadIdx.x;
  const int64_t chunk = blockIdx.x, group = chunk / per_group;
  const int64_t first = group * p.gate_rows + chunk % per_group * kGradRows;
  const int64_t last = min(min(first + kGradRows, (group + 1) * p.gate_rows), p.rows);
  const float inv_cols = 1.0f / float(p.cols);
  const MatrixRef gates{const_cast<void *>(p.gate), p.ld_gate, p.gate_bf16, 0};
  __shared__ __attribute__((aligned(16))) f32x4 sum_slots[NV > 1 ? 4 * NV * kLanes : 1];
  ColumnSums<NV> pre_sum, gate_sum;
  pre_sum.clear(sum_slots);
  gate_sum.clear(sum_slots + (NV > 1 ? 2 * NV * kLanes : 0));
  uint32_t col[NV];
  int n[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    col[v] = (uint32_t(v) * blockDim.x + tid) * 8;
    n[v] = max(0, min(8, int(p.cols) - int(col[v])));
  }
  Row<NV, BF16> dh, r, dr, y;
  if (first < last) {
    dh.fetch(p.dh, first, col, n);
    r.fetch(p.r, first, col, n);
    dr.fetch(p.dr, first, col, n);
    y.fetch(p.y, first, col, n);
  }
#pragma unroll 1
  for (int64_t row = first; row < last; ++row) {
    const int64_t next = min(row + 1, last - 1);  // past the last row: it again, not used
    float(*red)[kLanes / 64] = reds + 2 * (row & 1);
    float t[NV][8];
    if (p.dh.data != nullptr) {
      float m[NV][8], sum = 0.0f;
      const float f = p.pre_rstd[row];
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float w[8];
        weights8(p.pre_weight, p.weight_bf16 != 0, col[v], n[v], p.offset, w);
        dh.get(p.dh, row, col[v], n[v], v, t[v]);
        r.get(p.r, row, col[v], n[v], v, m[v]);
#pragma unroll
        for (int e = 0; e < 8; ++e) m[v][e] *= f;
        pre_sum.add(v, t[v], m[v]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          t[v][e] *= w[e];
          sum = __builtin_fmaf(t[v][e], m[v][e], sum);
        }
      }
      dh.fetch(p.dh, next, col, n);
      r.fetch(p.r, next, col, n);
      sum = group_sum(sum, red[0]) * inv_cols;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float d[8] = {};
        if (p.dr.data != nullptr) dr.get(p.dr, row, col[v], n[v], v, d);
#pragma unroll
        for (int e = 0; e < 8; ++e) t[v][e] = __builtin_fmaf(f, t[v][e] - m[v][e] * sum, d[e]);
        }
    } else {
#pragma unroll
      for (int v = 0; v < NV; ++v) dr.get(p.dr, row, col[v], n[v], v, t[v]);
    }
    dr.fetch(p.dr, next, col, n);
    if (p.dx.data != nullptr) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float dx[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) dx[e] = p.x_scale * t[v][e];
        store8(row_of(p.dx, is_bf16<BF16>(p.dx), row), is_bf16<BF16>(p.dx), col[v], n[v], dx);
      }
    }
    if (p.y.data == nullptr) continue;
    const float f = p.post_norm ? p.post_rstd[row] : 1.0f;
    float m[NV][8], sum = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float w[8], g[8];
      y.get(p.y, row, col[v], n[v], v, m[v]);
#pragma unroll
      for (int e = 0; e < 8; ++e) g[e] = w[e] = 1.0f;
      if (p.post_norm) weights8(p.post_weight, p.weight_bf16 != 0, col[v], n[v], p.offset, w);
      if (p.gate != nullptr) load8(row_of(gates, p.gate_bf16 != 0, group), p.gate_bf16 != 0, col[v], n[v], g);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        m[v][e] *= f;
        t[v][e] *= p.y_scale;
      }
      gate_sum.add(v, t[v], m[v]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        t[v][e] *= g[e] * w[e];
        sum = __builtin_fmaf(t[v][e], m[v][e], sum);
      }
    }
    y.fetch(p.y, next, col, n);
    if (p.dy.data == nullptr) continue;
    if (p.post_norm) {
      sum = group_sum(sum, red[1]) * inv_cols;
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) t[v][e] = f * (t[v][e] - m[v][e] * sum);
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) store8(row_of(p.dy, is_bf16<BF16>(p.dy), row), is_bf16<BF16>(p.dy), col[v], n[v], t[v]);
  }
  if (p.sums == nullptr) return;
  if (p.dpre != nullptr) {
#pragma unroll
    for (int v = 0; v < NV; ++v) pre_sum.store(p.sums + chunk * p.cols, v, col[v], n[v]);
  }
  if (p.dpost != nullptr || p.dgate != nullptr) {
#pragma unroll
    for (int v = 0; v < NV; ++v) gate_sum.store(p.sums + (chunks + chunk) * p.cols, v, col[v], n[v]);
  }
}

// The sum over i < count of a[i stride] in the workgroup's first 64 lanes: 64 columns
// a workgroup, four lanes a column, each every fourth row, then those four; always in
// that order.
__device__ __forceinline__ float column_sum(const float *a, int64_t count, int64_t stride, bool live, float *part) {
  float s = 0.0f;
  if (live) {
#pragma unroll 4
    for (int64_t i = threadIdx.x >> 6; i < count; i += 4) s += a[i * stride];
  }
  __syncthreads();
  part[threadIdx.x] = s;
  __syncthreads();
  const int l = threadIdx.x & 63;
  return (part[l] + part[64 + l]) + (part[128 + l] + part[192 + l]);
}

__device__ __forceinline__ float value_at(const void *p, bool bf16, int64_t at) {
  return bf16 ? bf16_to_f32(static_cast<const uint16_t *>(p)[at]) : static_cast<const float *>(p)[at];
}

// One group of gates a workgroup (and 64 columns): dgate, and S gate in the place of the group's first chunk.
__global__ __launch_bounds__(kThreads) void gate_grad_kernel(ResidualGradParams p, int64_t per_group, int64_t chunks, int64_t blocks_c) {
  __shared__ float part[kThreads];
  const int64_t group = int64_t(blockIdx.x) / blocks_c, c = int64_t(blockIdx.x) % blocks_c * 64 + (threadIdx.x & 63);
  float *a = p.sums + (chunks + group * per_group) * p.cols + c;
  const float s = column_sum(a, per_group, p.cols, c < p.cols, part);
  if (threadIdx.x >= 64 || c >= p.cols) return;
  if (p.dgate != nullptr) {
    const float w = p.post_norm && p.post_weight != nullptr ? p.offset + value_at(p.post_weight, p.weight_bf16 != 0, c) : 1.0f;
    float *d = p.dgate + group * p.ld_dgate + c;
    *d = p.accumulate ? *d + s * w : s * w;
  }
  *a = s * value_at(p.gate, p.gate_bf16 != 0, group * p.ld_gate + c);
}

// dw_pre from all chunks; dw_post from `post_count` rows of sums `post_stride` apart.
__global__ __launch_bounds__(kThreads) void weight_grad_kernel(ResidualGradParams p, int64_t chunks, int64_t post_count, int64_t post_stride) {
  __shared__ float part[kThreads];
  const int64_t c = int64_t(blockIdx.x) * 64 + (threadIdx.x & 63);
  const bool live = c < p.cols;
  if (p.dpre != nullptr) {
    const float s = column_sum(p.sums + c, chunks, p.cols, live, part);
    if (threadIdx.x < 64 && live) p.dpre[c] = p.accumulate ? p.dpre[c] + s : s;
  }
  if (p.dpost != nullptr) {
    const float s = column_sum(p.sums + chunks * p.cols + c, post_count, post_stride * p.cols, live, part);
    if (threadIdx.x < 64 && live) p.dpost[c] = p.accumulate ? p.dpost[c] + s : s;
  }
}

// Lanes and vectors of eight values a lane for a row.
struct RowShape {
  int lanes, vectors;
};
RowShape row_shape(int64_t cols) {
  int lanes = 64, vectors = 1;
  while (int64_t(lanes) * 8 < cols && lanes < kLanes) lanes *= 2;
  while (int64_t(lanes) * 8 * vectors < cols) vectors *= 2;
  return {lanes, vectors};
}

template <int NV>
hipError_t launch_grad_rows(const ResidualGradParams &p, bool bf16, int lanes, int64_t per_group, int64_t chunks, hipStream_t s) {
  const dim3 grid{unsigned(chunks)}, block{unsigned(lanes)};
  return bf16 ? klaunch(residual_grad_kernel<NV, true>, grid, block, 0, s, p, per_group, chunks)
              : klaunch(residual_grad_kernel<NV, false>, grid, block, 0, s, p, per_group, chunks);
}

bool all_bf16(std::initializer_list<const MatrixRef *> ms) {
  for (const MatrixRef *m : ms)
    if (m->data != nullptr && !m->bf16) return false;
  return true;
}

}  // namespace

hipError_t launch_residual_norm(const ResidualParams &p, hipStream_t s) {
  if (p.rows <= 0 || p.cols <= 0) return hipSuccess;
  const RowShape sh = row_shape(p.cols);
  if (sh.vectors > 2) return hipErrorInvalidValue;
  const bool bf16 = all_bf16({&p.x, &p.y, &p.r, &p.h});
  const int64_t most = ((int64_t(1) << 32) - 1) / sh.lanes;  // a launch has less than 2^32 lanes
  for (int64_t r0 = 0; r0 < p.rows; r0 += most) {
    ResidualParams q = p;
    q.row0 = r0;
    const dim3 grid{unsigned(std::min(most, p.rows - r0))}, block{unsigned(sh.lanes)};
    const hipError_t e = sh.vectors == 1 ? (bf16 ? klaunch(residual_norm_kernel<1, true>, grid, block, 0, s, q)
                                                 : klaunch(residual_norm_kernel<1, false>, grid, block, 0, s, q))
                                         : (bf16 ? klaunch(residual_norm_kernel<2, true>, grid, block, 0, s, q)
                                                 : klaunch(residual_norm_kernel<2, false>, grid, block, 0, s, q));
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_residual_grad(const ResidualGradParams &p, hipStream_t s) {
  if (p.cols <= 0) return hipSuccess;
  const int64_t per_group = (p.gate_rows + kGradRows - 1) / kGradRows, chunks = p.groups * per_group;
  if (chunks > 0) {
    const RowShape sh = row_shape(p.cols);
    const bool bf16 = all_bf16({&p.dr, &p.dh, &p.r, &p.y, &p.dx, &p.dy});
    const hipError_t e = sh.vectors == 1   ? launch_grad_rows<1>(p, bf16, sh.lanes, per_group, chunks, s)
                         : sh.vectors == 2 ? launch_grad_rows<2>(p, bf16, sh.lanes, per_group, chunks, s)
                                           : hipErrorInvalidValue;
    if (e != hipSuccess) return e;
  }
  const int64_t blocks_c = (p.cols + 63) / 64;
  int64_t post_count = chunks, post_stride = 1;
  if (p.gate != nullptr && p.groups > 0 && (p.dgate != nullptr || p.dpost != nullptr)) {
    const hipError_t e = klaunch(gate_grad_kernel, dim3(unsigned(p.groups * blocks_c)), dim3(kThreads), 0, s, p, per_group, chunks, blocks_c);
    if (e != hipSuccess) return e;
    post_count = p.groups;
    post_stride = per_group;
  }
  if (p.dpre == nullptr && p.dpost == nullptr) return hipSuccess;
  return klaunch(weight_grad_kernel, dim3(unsigned(blocks_c)), dim3(kThreads), 0, s, p, chunks, post_count, post_stride);
}

}  // namespace qe
