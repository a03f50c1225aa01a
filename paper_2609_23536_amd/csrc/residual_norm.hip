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
//     dx = x_scale t,   dw_pre = sum dh n
//     dy = f(y) (e - m mean(e m)),  e = t c,  c = y_scale gate (o + w_post)
// and with S = y_scale sum t m over the rows that share a row of gates:
//     dgate = S (o + w_post),   dw_post = sum over the gates' rows of S gate
// so one sum of columns serves both.
//
// Rows of more than 2048 columns are bound by memory (MI355X, 8192 x 8192 BF16: 86 us to r and
// row-wise codes, 5.5 TB/s, 98 to r and h; FP32 199, 5.4 TB/s; an FP32 stream with a BF16
// branch 151, 5.3 TB/s; the gradient 157, 5.1 TB/s, with its sums 167, FP32 323), and next by
// their vector instructions; rows of sixteen values a lane less so (4096 x 16384 BF16 110 and
// 221).  A workgroup takes one row after the other, each by a team of lanes that hold eight
// neighbouring values (or twice eight) of it in registers from the loads to the stores.
// With eight values a lane, what a column's weights and gates come to is kept from row to
// row.  BF16 rows are loaded a row ahead, before this one's sums are taken (the gradient's
// with eight values a lane only); others when they are used, or, in the gradient with eight
// values a lane, when their row begins.
#include "block_scale.h"

#include <algorithm>
#include <initializer_list>
#include <utility>

namespace qe {
namespace {

constexpr int kLanes = 1024;  // most lanes for a row

template <int CTRL>
__device__ __forceinline__ float add_dpp(float v) {
  return v + __uint_as_float(uint32_t(__builtin_amdgcn_mov_dpp(int(__float_as_uint(v)), CTRL, 0xf, 0xf, true)));
}
// Sum over an aligned group of 16 lanes, in all of them: lanes l ^ 1, l ^ 2, then 7 - l and 15 - l.
__device__ __forceinline__ float sum_lanes16(float v) { return add_dpp<0x140>(add_dpp<0x141>(add_dpp<0x4e>(add_dpp<0xb1>(v)))); }
// Sum over the wave, in all lanes.
__device__ __forceinline__ float wave_sum(float v) {
  v = sum_lanes16(v);
  uint32_t b = __float_as_uint(v);
  auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
  b = __float_as_uint(__uint_as_float(r[0]) + __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Sum over the team of 2^k (at most 16) waves that this wave is in, in all its lanes.
// `red`: one float per wave of the workgroup, which no sum before the last one has used
// (a lane may still be reading what that one left).  All waves of the workgroup come here.
__device__ __forceinline__ float team_sum(float v, float *red, int waves) {
  v = wave_sum(v);
  if (waves == 1) return v;
  const int wave = int(threadIdx.x) >> 6, l = int(threadIdx.x) & 15;
  if ((threadIdx.x & 63) == 0) red[wave] = v;
  __syncthreads();
  return sum_lanes16(l < waves ? red[(wave & -waves) + l] : 0.0f);
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

// A lane's columns of a row: NV times eight neighbouring ones, `lanes` lanes a row.
template <int NV>
struct Columns {
  uint32_t col[NV];
  int n[NV];  // those that exist
  __device__ __forceinline__ Columns(int lane, int lanes, int64_t cols) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      col[v] = uint32_t(v * lanes + lane) * 8;
      n[v] = max(0, min(8, int(cols) - int(col[v])));
    }
  }
};

// A row of an input.  kAhead: BF16, kept as it is stored from the moment it is fetched, a
// row before it is used.  kEarly: fetched as values when its row begins, so that the loads of
// a row wait for each other once.  kLate: loaded when it is used.
enum Fetch { kLate = 0, kEarly = 1, kAhead = 2 };
template <int NV, bool BF16, int WHEN>
struct Row {
  static_assert(BF16 || WHEN != kAhead, "four registers hold eight values");
  u32x4_in w[WHEN == kAhead ? NV : 1];
  float f[WHEN == kEarly ? NV : 1][8];
  __device__ __forceinline__ void fetch(const MatrixRef &m, int64_t row, const Columns<NV> &c) {
    if (WHEN == kLate || m.data == nullptr) return;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if constexpr (WHEN == kEarly) {
        load8(row_of(m, is_bf16<BF16>(m), row), is_bf16<BF16>(m), c.col[v], c.n[v], f[v]);
      } else if constexpr (WHEN == kAhead) {
        const uint16_t *p = reinterpret_cast<const uint16_t *>(row_of(m, true, row)) + c.col[v];
        if (c.n[v] >= 8) {
          w[v] = *reinterpret_cast<const u32x4_in *>(p);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            w[v][e] = (2 * e < c.n[v] ? uint32_t(p[2 * e]) : 0u) | (2 * e + 1 < c.n[v] ? uint32_t(p[2 * e + 1]) << 16 : 0u);
        }
      }
    }
  }
  __device__ __forceinline__ void get(const MatrixRef &m, int64_t row, const Columns<NV> &c, int v, float *out) const {
    if constexpr (WHEN == kAhead) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        out[2 * e] = __uint_as_float(w[v][e] << 16);
        out[2 * e + 1] = __uint_as_float(w[v][e] & 0xffff0000u);
      }
    } else if constexpr (WHEN == kEarly) {
#pragma unroll
      for (int e = 0; e < 8; ++e) out[e] = f[v][e];
    } else {
      load8(row_of(m, is_bf16<BF16>(m), row), is_bf16<BF16>(m), c.col[v], c.n[v], out);
    }
  }
};

// y_scale gate (o + w_post) of a vector of columns: what a row of gates makes of y's norm.
template <int NV, typename P>
__device__ __forceinline__ void branch_factors(const P &p, int64_t group, const Columns<NV> &c, int v, float *f) {
  const MatrixRef gates{const_cast<void *>(p.gate), p.ld_gate, p.gate_bf16, 0};
  float g[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = g[e] = 1.0f;
  if (p.post_norm) weights8(p.post_weight, p.weight_bf16 != 0, c.col[v], c.n[v], p.offset, f);
  if (p.gate != nullptr) load8(row_of(gates, p.gate_bf16 != 0, group), p.gate_bf16 != 0, c.col[v], c.n[v], g);
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] *= g[e] * p.y_scale;
}

// A workgroup takes rows blockIdx.x, + gridDim.x, .. of the launch.
// NV 1: 64 registers, so that a unit holds two workgroups of 1024 lanes.
template <int NV, bool BF16>
__global__ __launch_bounds__(kLanes, NV == 1 ? 8 : 4) void residual_norm_kernel(ResidualParams p, int row_lines) {
  __shared__ float reds[4][kLanes / 64];
  const int tid = threadIdx.x, waves = int(blockDim.x) >> 6;
  const float inv_cols = 1.0f / float(p.cols);
  const Columns<NV> c(tid, int(blockDim.x), p.cols);
  const bool has_x = p.x.data != nullptr, has_y = p.y.data != nullptr;
  // The columns' factors stay here, those of y's norm in registers and those of r's,
  // which 64 registers do not hold as well, in the lane's own 16-byte slots of LDS.
  constexpr bool KEEP = NV == 1;
  __shared__ __attribute__((aligned(16))) f32x4 slots[KEEP ? 2 * kLanes : 1];
  Row<NV, BF16, BF16 ? kAhead : kLate> x, y;
  x.fetch(p.x, blockIdx.x, c);
  y.fetch(p.y, blockIdx.x, c);
  float branch[NV][8];
  if constexpr (KEEP) {
    float w[8];
    weights8(p.pre_weight, p.weight_bf16 != 0, c.col[0], c.n[0], p.offset, w);
    slots[tid] = f32x4{w[0], w[1], w[2], w[3]};
    slots[kLanes + tid] = f32x4{w[4], w[5], w[6], w[7]};
  }
  const uint32_t gate_rows = uint32_t(p.gate_rows);
  uint32_t group = 0, group_end = 0;  // of the gates in `branch`
  int turn = 0;
#pragma unroll 1
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x, ++turn) {
    float(*red)[kLanes / 64] = reds + 2 * (turn & 1);
    const int64_t next = row + gridDim.x;
    if (has_y) {
      if (row >= group_end) {
        group = p.gate != nullptr ? uint32_t(row) / gate_rows : 0u;
        group_end = p.gate != nullptr ? (group + 1u) * gate_rows : 0xffffffffu;
        if constexpr (KEEP) branch_factors<NV>(p, group, c, 0, branch[0]);
      }
    }
    float r[NV][8];
    auto add_x = [&](int v) {  // r = x_scale x + r
      float f[8];
      x.get(p.x, row, c, v, f);
#pragma unroll
      for (int e = 0; e < 8; ++e) r[v][e] = __builtin_fmaf(p.x_scale, f[e], r[v][e]);
    };
    if (has_y) {
#pragma unroll
      for (int v = 0; v < NV; ++v) y.get(p.y, row, c, v, r[v]);
      if (next < p.rows) y.fetch(p.y, next, c);
      float f = 1.0f;
      if (p.post_norm) {
        float sum = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(r[v][e], r[v][e], sum);
        f = 1.0f / __builtin_sqrtf(team_sum(sum, red[0], waves) * inv_cols + p.post_eps);
        if (tid == 0 && p.post_rstd != nullptr) p.post_rstd[row] = f;
      }
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        if constexpr (!KEEP) branch_factors<NV>(p, group, c, v, branch[v]);
#pragma unroll
        for (int e = 0; e < 8; ++e) r[v][e] = r[v][e] * f * branch[v][e];
        if (has_x) add_x(v);
      }
    } else {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        x.get(p.x, row, c, v, r[v]);
#pragma unroll
        for (int e = 0; e < 8; ++e) r[v][e] *= p.x_scale;
      }
    }
    if (next < p.rows) x.fetch(p.x, next, c);
    if (p.r.data != nullptr) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        store8(row_of(p.r, is_bf16<BF16>(p.r), row), is_bf16<BF16>(p.r), c.col[v], c.n[v], r[v]);
        if (is_bf16<BF16>(p.r)) {
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            const uint32_t w = bf16x2_bits(r[v][e], r[v][e + 1]);
            r[v][e] = __uint_as_float(w << 16);
            r[v][e + 1] = __uint_as_float(w & 0xffff0000u);
          }
        }
      }
    }
    if (!p.pre_norm) continue;
    float sum = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(r[v][e], r[v][e], sum);
    const float f = 1.0f / __builtin_sqrtf(team_sum(sum, red[1], waves) * inv_cols + p.pre_eps);
    if (tid == 0 && p.pre_rstd != nullptr) p.pre_rstd[row] = f;
    if (p.h.data == nullptr && p.row.data == nullptr) continue;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float h[8], w[8];
      if constexpr (KEEP) {
        const f32x4 lo = slots[tid], hi = slots[kLanes + tid];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = e < 4 ? lo[e % 4] : hi[e % 4];
      } else {
        weights8(p.pre_weight, p.weight_bf16 != 0, c.col[v], c.n[v], p.offset, w);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) h[e] = r[v][e] * f * w[e];
      if (p.h.data != nullptr) store8(row_of(p.h, is_bf16<BF16>(p.h), row), is_bf16<BF16>(p.h), c.col[v], c.n[v], h);
      if (p.row.data != nullptr) {
        // (columns past the last one are 0, or NaN where the whole row is)
        const float a = max_lanes16(nan_max(amax4(f32x4{h[0], h[1], h[2], h[3]}), amax4(f32x4{h[4], h[5], h[6], h[7]})));
        uint8_t *dst = (p.row.data + row * p.row.ld) + c.col[v];
        const uint32_t byte = p.row.fmt == 0 ? block_byte<0>(a) : block_byte<1>(a);
        const float step = block_step(byte);
        if (p.row.fmt == 0)
          store_codes8(dst, c.n[v], block_codes<0>(h, step), block_codes<0>(h + 4, step), row_lines != 0);
        else
          store_codes8(dst, c.n[v], block_codes<1>(h, step), block_codes<1>(h + 4, step), row_lines != 0);
        if ((tid & 15) == 0 && c.n[v] > 0) (p.row.exps + row * p.row.ld_exps)[c.col[v] / kBlock] = uint8_t(byte);
      }
    }
  }
}

// Column sums of a lane's columns: in registers with eight of them, in LDS (the lane's
// own 16-byte slots) with sixteen, where 128 registers a lane do not hold them.
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
  // With one vector: the sums of all teams of `lanes` lanes, in the first team's, in their order.
  __device__ __forceinline__ void join(int lanes) {
    if constexpr (!kInLds) {
      lds[0] = reg[0];
      lds[kLanes] = reg[1];
      __syncthreads();
      if (int(threadIdx.x) < lanes)
        for (int at = lanes; at < int(blockDim.x); at += lanes) {
          reg[0] += lds[at];
          reg[1] += lds[kLanes + at];
        }
    }
  }
  __device__ __forceinline__ void store(float *row, int v, uint32_t col, int n, float scale) const {
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = scale * (kInLds ? lds[(2 * v + e / 4) * kLanes][e % 4] : reg[kInLds ? 0 : e / 4][e % 4]);
    store8(row, false, col, n, f);
  }
};

// Where the columns are summed by a kernel of their own (column_sums_kernel), the mean of
// d n over row i of a chunk of kGradRows waits for it in the workspace, where the chunk's
// sums of a block of columns will be, once for each block: the first eight rows' in the
// block's sums of dh n, the others' in those of t m.
constexpr int kSumCols = 512, kHalf = int(kGradRows) / 2;
__device__ __forceinline__ float *waiting(const ResidualGradParams &p, int64_t chunks, int64_t chunk, int block, int i) {
  return p.sums + ((i < kHalf ? 0 : chunks) + chunk) * p.cols + block * kSumCols + i % kHalf;
}

// Chunks of up to chunk_rows rows, `per_group` of them for each group of gate_rows rows;
// a chunk is a workgroup, whose teams of `lanes` lanes take every so manyth row of it.
// sum_chunks > 0: no column sums, but each row's mean left for column_sums_kernel, whose
// chunks those are (sum_group of them in a group).
template <int NV, bool BF16>
__global__ __launch_bounds__(kLanes) void residual_grad_kernel(ResidualGradParams p, int64_t per_group, int64_t chunks, int64_t chunk_rows, int lanes,
                                                               int64_t sum_chunks, int64_t sum_group) {
  __shared__ __attribute__((aligned(16))) float reds[4][kLanes / 64];
  __shared__ __attribute__((aligned(16))) f32x4 sum_slots[4 * NV * kLanes];
  const int tid = threadIdx.x, waves = lanes >> 6, team = tid / lanes, teams = int(blockDim.x) / lanes;
  const int64_t chunk = blockIdx.x, group = blockIdx.x / uint32_t(per_group);
  const int64_t first = group * p.gate_rows + (chunk - group * per_group) * chunk_rows;
  const int64_t last = min(min(first + chunk_rows, (group + 1) * p.gate_rows), p.rows);
  const float inv_cols = 1.0f / float(p.cols);
  const Columns<NV> c(tid % lanes, lanes, p.cols);
  ColumnSums<NV> pre_sum, gate_sum;
  pre_sum.clear(sum_slots);
  gate_sum.clear(sum_slots + 2 * NV * kLanes);
  // The columns' factors stay in registers, and rows are loaded ahead of their use, where they hold it.
  constexpr bool KEEP = NV == 1;
  constexpr int WHEN = NV > 1 ? kLate : (BF16 ? kAhead : kEarly);
  Row<NV, BF16, WHEN> dh, r, dr, y;
  const int64_t mine = min(first + team, last - 1);  // a team without a row: the last one again, not counted
  auto fetch_all = [&](int64_t row) {
    dh.fetch(p.dh, row, c);
    r.fetch(p.r, row, c);
    dr.fetch(p.dr, row, c);
    y.fetch(p.y, row, c);
  };
  if (WHEN == kAhead && first < last) fetch_all(mine);
  float pre_w[NV][8], branch[NV][8];
  auto pre_weights = [&](int v) { weights8(p.pre_weight, p.weight_bf16 != 0, c.col[v], c.n[v], p.offset, pre_w[v]); };
  if constexpr (KEEP) {
    pre_weights(0);
    branch_factors<NV>(p, group, c, 0, branch[0]);
  }
  int turn = 0;
#pragma unroll 1
  for (int64_t row0 = first; row0 < last; row0 += teams, ++turn) {
    const bool live = row0 + team < last;
    const int64_t row = live ? row0 + team : last - 1, next = min(row + teams, last - 1);
    float(*red)[kLanes / 64] = reds + 2 * (turn & 1);
    float t[NV][8];
    if (WHEN == kEarly) fetch_all(row);
    if (p.dh.data != nullptr) {
      float m[NV][8], sum = 0.0f;
      const float f = p.pre_rstd[row];
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        dh.get(p.dh, row, c, v, t[v]);
        r.get(p.r, row, c, v, m[v]);
#pragma unroll
        for (int e = 0; e < 8; ++e) m[v][e] *= f;
        if (live && sum_chunks == 0) pre_sum.add(v, t[v], m[v]);
        if constexpr (!KEEP) pre_weights(v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          t[v][e] *= pre_w[v][e];
          sum = __builtin_fmaf(t[v][e], m[v][e], sum);
        }
      }
      if (WHEN == kAhead) {
        dh.fetch(p.dh, next, c);
        r.fetch(p.r, next, c);
      }
      sum = team_sum(sum, red[0], waves) * inv_cols;
      if (sum_chunks > 0 && live) {
        const int64_t in_group = row - group * p.gate_rows;
        const int block = tid - team * lanes;
        if (int64_t(block) * kSumCols < p.cols)
          *waiting(p, sum_chunks, group * sum_group + in_group / kGradRows, block, int(in_group % kGradRows)) = sum;
      }
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float d[8] = {};
        if (p.dr.data != nullptr) dr.get(p.dr, row, c, v, d);
#pragma unroll
        for (int e = 0; e < 8; ++e) t[v][e] = __builtin_fmaf(f, t[v][e] - m[v][e] * sum, d[e]);
      }
    } else {
#pragma unroll
      for (int v = 0; v < NV; ++v) dr.get(p.dr, row, c, v, t[v]);
    }
    if (WHEN == kAhead) dr.fetch(p.dr, next, c);
    if (p.dx.data != nullptr && live) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float dx[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) dx[e] = p.x_scale * t[v][e];
        store8(row_of(p.dx, is_bf16<BF16>(p.dx), row), is_bf16<BF16>(p.dx), c.col[v], c.n[v], dx);
      }
    }
    if (p.y.data == nullptr) continue;
    const float f = p.post_norm ? p.post_rstd[row] : 1.0f;
    float m[NV][8], sum = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      y.get(p.y, row, c, v, m[v]);
#pragma unroll
      for (int e = 0; e < 8; ++e) m[v][e] *= f;
      if (live && sum_chunks == 0) gate_sum.add(v, t[v], m[v]);
      if constexpr (!KEEP) branch_factors<NV>(p, group, c, v, branch[v]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        t[v][e] *= branch[v][e];
        sum = __builtin_fmaf(t[v][e], m[v][e], sum);
      }
    }
    if (WHEN == kAhead) y.fetch(p.y, next, c);
    if (p.dy.data == nullptr) continue;
    if (p.post_norm) {
      sum = team_sum(sum, red[1], waves) * inv_cols;
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) t[v][e] = f * (t[v][e] - m[v][e] * sum);
    }
    if (live) {
#pragma unroll
      for (int v = 0; v < NV; ++v) store8(row_of(p.dy, is_bf16<BF16>(p.dy), row), is_bf16<BF16>(p.dy), c.col[v], c.n[v], t[v]);
    }
  }
  if (p.sums == nullptr || sum_chunks > 0) return;
  if (teams > 1) {
    pre_sum.join(lanes);
    gate_sum.join(lanes);
    if (team != 0) return;
  }
  if (p.dpre != nullptr) {
#pragma unroll
    for (int v = 0; v < NV; ++v) pre_sum.store(p.sums + chunk * p.cols, v, c.col[v], c.n[v], 1.0f);
  }
  if (p.dpost != nullptr || p.dgate != nullptr) {
#pragma unroll
    for (int v = 0; v < NV; ++v) gate_sum.store(p.sums + (chunks + chunk) * p.cols, v, c.col[v], c.n[v], p.y_scale);
  }
}

// The column sums of a chunk of kGradRows rows for a block of kSumCols columns: a wave
// per row, which computes dh n and t m again from the inputs and the row's mean, then the
// waves' in their order.
template <bool BF16>
__global__ __launch_bounds__(64 * kGradRows) void column_sums_kernel(ResidualGradParams p, int64_t per_group, int64_t chunks, int blocks) {
  __shared__ __attribute__((aligned(16))) f32x4 slots[kGradRows][4 * 64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  const int64_t chunk = blockIdx.x / unsigned(blocks), group = chunk / per_group;
  const int block = int(blockIdx.x % unsigned(blocks));
  const int64_t row = group * p.gate_rows + (chunk - group * per_group) * kGradRows + wave;
  const bool live = row < min((group + 1) * p.gate_rows, p.rows);
  Columns<1> c(lane, 64, p.cols - block * kSumCols);
  c.col[0] += uint32_t(block) * kSumCols;
  const bool gates = p.y.data != nullptr && (p.dpost != nullptr || p.dgate != nullptr);
  float pre[8] = {}, gate[8] = {};
  if (live) {
    Row<1, BF16, BF16 ? kAhead : kEarly> dh, r, dr, y;
    dh.fetch(p.dh, row, c);
    r.fetch(p.r, row, c);
    if (gates) {
      dr.fetch(p.dr, row, c);
      y.fetch(p.y, row, c);
    }
    float t[8] = {};
    if (gates && p.dr.data != nullptr) dr.get(p.dr, row, c, 0, t);
    if (p.dh.data != nullptr) {
      float d[8], m[8], w[8];
      const float f = p.pre_rstd[row], mean = *waiting(p, chunks, chunk, block, wave);
      dh.get(p.dh, row, c, 0, d);
      r.get(p.r, row, c, 0, m);
      weights8(p.pre_weight, p.weight_bf16 != 0, c.col[0], c.n[0], p.offset, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        m[e] *= f;
        pre[e] = d[e] * m[e];
        t[e] = __builtin_fmaf(f, d[e] * w[e] - m[e] * mean, t[e]);
      }
    }
    if (gates) {
      float m[8];
      const float f = p.post_norm ? p.post_rstd[row] : 1.0f;
      y.get(p.y, row, c, 0, m);
#pragma unroll
      for (int e = 0; e < 8; ++e) gate[e] = t[e] * (m[e] * f);
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    slots[wave][64 * h + lane] = f32x4{pre[4 * h], pre[4 * h + 1], pre[4 * h + 2], pre[4 * h + 3]};
    slots[wave][64 * (2 + h) + lane] = f32x4{gate[4 * h], gate[4 * h + 1], gate[4 * h + 2], gate[4 * h + 3]};
  }
  __syncthreads();  // (every wave has read its row's mean by now)
  if (threadIdx.x >= 256) return;
  f32x4 s = slots[0][threadIdx.x];
#pragma unroll
  for (int w = 1; w < int(kGradRows); ++w) s += slots[w][threadIdx.x];
  const bool of_gate = threadIdx.x >= 128;
  const int at = 8 * lane + 4 * (wave & 1), n = int(min(int64_t(4), p.cols - block * kSumCols - at));
  float *out = p.sums + ((of_gate ? chunks : 0) + chunk) * p.cols + block * kSumCols + at;
  const float scale = of_gate ? p.y_scale : 1.0f;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < n) out[e] = scale * s[e];
}

// The sum over i < count of a[i stride], a column a lane, in their order.
constexpr int kSumWaves = 16;
__device__ __forceinline__ float column_sum(const float *a, int64_t count, int64_t stride, int64_t first = 0, int step = 1) {
  float s = 0.0f;
#pragma unroll 8
  for (int64_t i = first; i < count; i += step) s += a[i * stride];
  return s;
}

// The waves' sums, in their order, in the first one.
__device__ __forceinline__ float join_waves(float s, float *part) {
  __syncthreads();  // the last sum's parts have been read
  part[threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.x < 64) {
#pragma unroll
    for (int w = 1; w < kSumWaves; ++w) s += part[64 * w + threadIdx.x];
  }
  return s;
}

__device__ __forceinline__ float value_at(const void *p, bool bf16, int64_t at) {
  return bf16 ? bf16_to_f32(static_cast<const uint16_t *>(p)[at]) : static_cast<const float *>(p)[at];
}

// How the chunks of groups are added up.
enum GroupSums {
  kByWorkgroup,  // a group, for 64 columns, is a workgroup's
  kByWave,       // .. a wave's
  kTogether,     // .. a wave's, and all groups a workgroup's, which adds up dw_post
};

// Blocks of 64 columns: first those of dw_pre (pre_blocks of them, or none), then those of
// S (post_blocks: of each group, or kTogether of all): dgate, and dw_post where one
// workgroup has all of it, else S gate in the place of the group's first chunk.  A launch
// holds less than 2^32 lanes: a workgroup may have to take more than one block.
__global__ __launch_bounds__(64 * kSumWaves) void column_grad_kernel(ResidualGradParams p, int64_t per_group, int64_t chunks, int64_t blocks_c,
                                                                     int64_t pre_blocks, int64_t post_blocks, int how) {
  __shared__ float part[64 * kSumWaves];
  const int64_t per_workgroup = how == kByWave ? kSumWaves : 1, total = pre_blocks + (post_blocks + per_workgroup - 1) / per_workgroup;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  auto of_group = [&](int64_t group, int64_t c, float s) {  // S -> S gate, and dgate
    if (p.dgate != nullptr) {
      const float w = p.post_norm && p.post_weight != nullptr ? p.offset + value_at(p.post_weight, p.weight_bf16 != 0, c) : 1.0f;
      float *d = p.dgate + group * p.ld_dgate + c;
      *d = p.accumulate ? *d + s * w : s * w;
    }
    return p.gate != nullptr ? s * value_at(p.gate, p.gate_bf16 != 0, group * p.ld_gate + c) : s;
  };
#pragma unroll 1
  for (int64_t at = blockIdx.x; at < total; at += gridDim.x) {
    const bool pre = at < pre_blocks;
    const int64_t block = pre ? at : (at - pre_blocks) * per_workgroup + (how == kByWave ? wave : 0);
    const int64_t group = block / blocks_c, c = block % blocks_c * 64 + lane;
    const bool live = c < p.cols && (pre || block < post_blocks);
    float *a = p.sums + (pre ? 0 : chunks * p.cols) + c, s = 0.0f;
    if (pre) {
      s = join_waves(live ? column_sum(a, chunks, p.cols, wave, kSumWaves) : 0.0f, part);
    } else if (how == kTogether) {
      if (live)
        for (int64_t g = wave; g < p.groups; g += kSumWaves) s += of_group(g, c, column_sum(a + g * per_group * p.cols, per_group, p.cols));
      s = join_waves(s, part);
    } else {
      a += group * per_group * p.cols;
      if (how == kByWave)
        s = live ? column_sum(a, per_group, p.cols) : 0.0f;
      else
        s = join_waves(live ? column_sum(a, per_group, p.cols, wave, kSumWaves) : 0.0f, part);
    }
    if (!live || ((pre || how != kByWave) && wave != 0)) continue;
    if (!pre && how != kTogether) s = of_group(group, c, s);
    float *out = pre ? p.dpre : p.dpost;
    if (out == nullptr) continue;
    if (!pre && how != kTogether && p.groups > 1)
      *a = s;
    else
      out[c] = p.accumulate ? out[c] + s : s;
  }
}

// dw_post from the groups' rows.
__global__ __launch_bounds__(64 * kSumWaves) void post_grad_kernel(ResidualGradParams p, int64_t per_group, int64_t chunks) {
  __shared__ float part[64 * kSumWaves];
  const int64_t c = int64_t(blockIdx.x) * 64 + (threadIdx.x & 63);
  const float *a = p.sums + chunks * p.cols + c;
  const float s = join_waves(c < p.cols ? column_sum(a, p.groups, per_group * p.cols, threadIdx.x >> 6, kSumWaves) : 0.0f, part);
  if (threadIdx.x < 64 && c < p.cols) p.dpost[c] = p.accumulate ? p.dpost[c] + s : s;
}

// Chunks of a group that one wave adds up.  MI355X, us for the whole gradient, sixteen
// waves a group / one: 8192 x 8192 with a row of gates for 256 rows (16 chunks) 191 / 173,
// 64 rows (4) 261 / 182, 16 rows (1) 545 / 224; 2048 x 2048, 128 rows (8) 24.4 / 23.0.
constexpr int64_t kFewChunks = 16;
constexpr int64_t kFewGroups = 256;  // (sixteen a wave) that are added up together

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

bool all_bf16(std::initializer_list<const MatrixRef *> ms) {
  for (const MatrixRef *m : ms)
    if (m->data != nullptr && !m->bf16) return false;
  return true;
}

// Few chunks of 16 rows leave most units idle, and rows of more than two thousand columns
// then follow each other in teams of half a workgroup or more: the columns are summed by a
// kernel of their own, which reads the inputs (in the caches by then) once more.  MI355X,
// us, sums with the rows / apart: 64 x 8192 37.7 / 15.5, 512 x 8192 43 / 24, 1280 x 8192 (80
// chunks) 62 / 52, 1000 x 2730 FP32 37.6 / 33.5, but 1280 x 4096 27.5 / 29.4, 2048 x 8192
// (128) 68 / 77; 512 x 2048 16.4 / 15.9, 64 x 1024 12.6 / 14.3.  A block's sums have room
// for the means of half a chunk's rows from eight columns on, and in place the inputs are
// gone by then.
bool sums_apart(const ResidualGradParams &p, int64_t chunks) {
  for (const MatrixRef *out : {&p.dx, &p.dy})
    for (const MatrixRef *in : {&p.dr, &p.dh, &p.r, &p.y})
      if (out->data != nullptr && out->data == in->data) return false;
  return chunks * 3 <= compute_units() && p.cols > 2048 && (p.cols % kSumCols == 0 || p.cols % kSumCols >= kHalf);
}

}  // namespace

hipError_t launch_residual_norm(const ResidualParams &p, hipStream_t s) {
  if (p.rows <= 0 || p.cols <= 0) return hipSuccess;
  const RowShape sh = row_shape(p.cols);
  if (sh.vectors > 2) return hipErrorInvalidValue;
  const bool bf16 = all_bf16({&p.x, &p.y, &p.r, &p.h});
  // 2048 lanes a unit, and each workgroup the rows it then has.  A unit holds them all with
  // eight values a lane and more than 2048 columns; half of them with sixteen (97 registers).
  // Of shorter rows it holds four workgroups, by the 32 KB that `slots` has for any number of
  // lanes, and the rest follow: MI355X, us, 16384 rows of BF16 with both norms, and the bytes
  // at 6.28 TB/s: 128 columns 42 / 2.7, 512 45 / 10.7, 1024 47 / 21.4, 2048 53 / 42.7, 4096
  // 101 / 85.5.
  const int64_t most = int64_t(compute_units()) * (2048 / sh.lanes);
  const dim3 grid{unsigned(std::min(p.rows, most))}, block{unsigned(sh.lanes)};
  const int lines = whole_lines(p.row) ? 1 : 0;
  return klaunch(sh.vectors == 1 ? (bf16 ? residual_norm_kernel<1, true> : residual_norm_kernel<1, false>)
                                 : (bf16 ? residual_norm_kernel<2, true> : residual_norm_kernel<2, false>),
                 grid, block, 0, s, p, lines);
}

hipError_t launch_residual_grad(const ResidualGradParams &p, hipStream_t s) {
  if (p.cols <= 0) return hipSuccess;
  int64_t per_group = 1, chunks = 0;
  if (p.rows > 0) {
    const RowShape sh = row_shape(p.cols);
    if (sh.vectors > 2) return hipErrorInvalidValue;
    const bool bf16 = all_bf16({&p.dr, &p.dh, &p.r, &p.y, &p.dx, &p.dy});
    // A unit holds one workgroup: as many chunks as units, or a few less where groups share
    // them (a chunk more than units is another round), of 16 rows at least where they leave
    // sums, which the workspace's size allows for.  MI355X, us, BF16 8192 x 8192 in 3, 5 and 7
    // groups, a chunk more / less: 263, 261, 264 / 178, 192, 182; 4096 x 8192 in 3: 142 / 99.
    const int64_t units = compute_units(), smallest = (p.gate_rows + kGradRows - 1) / kGradRows;
    const bool own_sums = p.sums != nullptr && sums_apart(p, smallest * p.groups);
    auto chunks_of = [&](int64_t least) {  // rows a chunk, and chunks a group
      const int64_t most = (p.gate_rows + least - 1) / least, n = std::min(most, std::max<int64_t>(units / p.groups, 1));
      const int64_t rows = (p.gate_rows + n - 1) / n;
      return std::make_pair(rows, (p.gate_rows + rows - 1) / rows);
    };
    const auto [chunk_rows, in_group] = chunks_of(p.sums != nullptr && !own_sums ? kGradRows : 1);
    const int teams = int(std::min<int64_t>(kLanes / sh.lanes, chunk_rows));
    const dim3 grid{unsigned(p.groups * in_group)}, block{unsigned(sh.lanes * teams)};
    per_group = own_sums ? smallest : in_group;
    chunks = p.groups * per_group;
    const int64_t apart = own_sums ? chunks : 0;
    auto rows_kernel = [&](auto *kernel) {
      return klaunch(kernel, grid, block, 0, s, p, in_group, p.groups * in_group, chunk_rows, sh.lanes, apart, smallest);
    };
    hipError_t e = sh.vectors == 1 ? rows_kernel(bf16 ? residual_grad_kernel<1, true> : residual_grad_kernel<1, false>)
                                   : rows_kernel(bf16 ? residual_grad_kernel<2, true> : residual_grad_kernel<2, false>);
    if (e == hipSuccess && own_sums) {
      const int blocks = int((p.cols + kSumCols - 1) / kSumCols);
      e = klaunch(bf16 ? column_sums_kernel<true> : column_sums_kernel<false>, dim3(unsigned(chunks * blocks)), dim3(64 * kGradRows), 0, s, p,
                  per_group, chunks, blocks);
    }
    if (e != hipSuccess) return e;
  }
  const int64_t blocks_c = (p.cols + 63) / 64, pre_blocks = p.dpre != nullptr ? blocks_c : 0;
  // (without rows one group of no chunks, whose sums are zero)
  const bool post = p.dpost != nullptr || (p.dgate != nullptr && p.groups > 0);
  const bool together = p.dpost != nullptr && p.groups > 1 && p.groups <= kFewGroups && per_group <= kFewChunks;
  const int how = per_group > kFewChunks ? kByWorkgroup : together ? kTogether : kByWave;
  const int64_t post_blocks = !post ? 0 : together ? blocks_c : std::max<int64_t>(p.groups, 1) * blocks_c;
  if (pre_blocks + post_blocks == 0) return hipSuccess;
  ResidualGradParams q = p;
  if (p.groups == 0) q.dgate = nullptr, q.gate = nullptr;
  const dim3 block(64 * kSumWaves);
  const int64_t blocks = pre_blocks + (how == kByWave ? (post_blocks + kSumWaves - 1) / kSumWaves : post_blocks), most = (int64_t(1) << 22) - 1;
  hipError_t e = klaunch(column_grad_kernel, dim3(unsigned(std::min(blocks, most))), block, 0, s, q, chunks > 0 ? per_group : 0, chunks, blocks_c,
                         pre_blocks, post_blocks, how);
  if (e == hipSuccess && p.groups > 1 && p.dpost != nullptr && !together)
    e = klaunch(post_grad_kernel, dim3(unsigned(blocks_c)), block, 0, s, p, per_group, chunks);
  return e;
}

}  // namespace qe
