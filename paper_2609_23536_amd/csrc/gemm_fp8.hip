// FP8 GEMM for the three products of the split linear (gfx950 MFMA).
//
// §3.2 of the paper: F computes Y = X W^T, dI computes dX = dY W, and the
// deferred dW computes dW = dY^T X, each on FP8-quantized operands.  With the
// quantizer writing every operand both row-wise and transposed, all three are
// the same "TN" product with both operands contiguous along the reduction:
//     D[i][j] = 2^(ea + eb) * sum_r A[i][r] B[j][r]
// where 2^ea, 2^eb are the operands' scale inverses (powers of two, so the
// rescale is exact; other values are multiplied in as they are).  The epilogue
// stores D (FP32 or BF16), or adds it to an FP32 destination in place: the direct
// placement of dW into its slice of the flat main-gradient buffer (§3.4), with no
// staging copy.
//
// gemm_tn_w4_kernel serves the large tiles, 256 x 256 x 128 (and 256 x 224,
// 256 x 192, 192 x 256); gemm_ring.hip the small ones.  Every shape uses
// v_mfma_f32_16x16x128_f8f6f4 with the same assignment of reduction bytes to
// lanes and accumulates each output element in the same order, so all give the
// same bits.  Four waves (one per SIMD) on a 2 x 2 grid, each a 128 x 128
// sub-tile of 8 x 8 MFMA blocks.  A K tile's 64 MFMAs run in two phases; every
// fragment read or LDS-bound load is issued right after an MFMA, in a fixed
// order (sched_barrier), so the MFMA pipe stays busy in the single wave, and
// the LDS-bound loads are branch-free (two instructions each) because a single
// wave issues at most one instruction per four cycles, eight per MFMA.  The K
// loop is rotated so that its back-edge sits at the stage barrier, where all
// LDS reads have completed; the compiler can then wait for fragment reads one
// by one instead of draining them at the loop head.  The epilogue goes through
// LDS so every store instruction writes whole row runs (512-byte FP32 runs;
// BF16 values are rounded first and go as 256-byte runs).
// Operand formats (E4M3 or E5M2) are chosen per call.  K tiles are
// double-buffered in LDS and filled by LDS-bound global loads
// (global_load_lds_dwordx4: no register staging, no LDS store instructions)
// issued a K tile ahead; each wave waits for its own loads and a barrier
// publishes the stage.  The 4-wave kernel splits a K tile's loads: the B part
// goes into a stage's B half as soon as every wave holds the B fragments of
// the tile that stage held (during phase A, a K step and a half before it is
// read), the A part in the first half of phase B; a second barrier per K step
// marks the B half free.  (Measured on MI355X: against all loads spread over
// phase B, the Llama-3-70B stage's GEMMs 4% faster, products whose operands
// stream from HBM up to 8%.)  LDS rows are 128 bytes, their 16-byte chunks
// XOR-swizzled by row (row_swizzle) so that a fragment read meets no bank
// conflict, and since fragments start on multiples of 16 rows, every fragment
// of a wave is one base address plus a constant.  The LDS-bound loads are inline
// assembly: the compiler's own form makes it wait for them before every LDS
// read, serialising the loads with the MFMA work.  Rows past M / N are
// clamped to the last row (their results are never stored), so only the last,
// partial K tile needs masking; it goes through registers.
//
// MFMA operand order: the B fragment is passed as source A and the A fragment
// as source B, so each lane ends up holding four consecutive output columns of
// one output row and the epilogue stores 16 bytes per lane.  Within a lane the
// 32 reduction bytes of a fragment come from the same positions for A and B,
// so any fixed assignment of reduction indices to MFMA slots gives the same
// dot products.
//
// Determinism: no atomics and no split reduction; the same inputs produce the
// same bits, which the split-vs-full-backward check relies on.
#include "gemm_loops.h"
#include "scale_update.h"

namespace qe {
namespace {

// 256 x 256 x 128 tile (also 256 x 224, 256 x 192 and 192 x 256), four waves
// (one per SIMD) on a 2 x 2 grid, each wave a TM x TN sub-tile of 16 x 16 blocks of
// v_mfma_f32_16x16x128_f8f6f4, one MFMA per block per K tile.  (On random FP8
// operands this MFMA sustains about a third more throughput than the 32 x 32 x
// 64 one on MI355X, which draws more power per FLOP; with constant operands
// the two are equal.)
// A K tile's MFMAs run in two phases of I/2 block rows each:
//   phase A (block rows 0 .. I/2-1, column-major): uses A fragments
//     0 .. I/2-1 and every B fragment; reads A fragments I/2 .. I-1 of the
//     same tile; issues the B part of the LDS-bound loads of the tile two K
//     tiles ahead into this stage's B half;
//   phase B (block rows I/2 .. I-1, column-major): each B fragment's last use
//     is followed by the read of the next tile's B fragment into the same
//     registers, and the next tile's A fragments 0 .. I/2-1 are read too; the
//     A part of the loads of the tile after next is issued in its first half.
// So all of tile t is read by the end of its phase A, where the stage barrier
// sits: it frees tile t's A half for the A part of tile t+2 and publishes tile
// t+1.  A second barrier, after phase B, marks the B half of tile t+1's stage
// free once every wave holds tile t+1's B fragments, so phase A of tile t+1
// loads tile t+3's B part there: a K step and a half of latency budget for
// the B part, about a phase for the A part.  Fragment registers: I + J
// fragments of 8 VGPRs, no second set.  The K loop is rotated (phase B of tile t, then phase A of tile t+1)
// so its back-edge sits at the barrier, where every LDS read has completed;
// the waits for fragment reads inside an iteration can then be partial.
template <int FA, int FB, int OUT, int BM, int BN>
__global__ __launch_bounds__(256) void gemm_tn_w4_kernel(GemmParams g, int tiles_m, int tiles_n, int vec_ok,
                                                         UpdateParams upd) {
  static_assert((BM == 256 || BM == 192) && (BN == 256 || BN == 224 || BN == 192), "tile sizes");
  constexpr int NW = 4, TM = BM / 2, TN = BN / 2;
  constexpr int I = TM / 16, J = TN / 16;    // 16 x 16 MFMA blocks per wave sub-tile
  constexpr int CHA = BM / 32, CHB = BN / 32;  // 16-byte LDS-bound loads per lane per K tile
  constexpr int STAGE = (BM + BN) * BK;
  constexpr int EP = TN + 4;                 // epilogue staging row, in floats (padded)
  static_assert(NW * 32 * EP * 4 <= 2 * STAGE, "epilogue staging fits in the stages");
  // two K stages, then one 1 KB block per wave that absorbs the loads issued
  // past the last full K tile (so the loop issues them unconditionally)
  __shared__ __attribute__((aligned(16))) uint8_t smem[2 * STAGE + NW * 1024];
  static_assert(sizeof(smem) >= (kMaxHistory + kUpdateThreads / 64) * 4, "history staging fits in the stages");

  // Workgroups past the tiles (dispatched last) run the delayed scale update
  // of the action's roles beside the tiles: the tiles read the scale_inv
  // snapshots, never the live scales this update writes.
  if (int(blockIdx.x) >= tiles_m * tiles_n) {
    const int r = int(blockIdx.x) - tiles_m * tiles_n;
    uint32_t *hs = reinterpret_cast<uint32_t *>(smem);
    scale_update_role(upd.m[r], r == 0 ? upd.token : nullptr, hs, hs + kMaxHistory);
    return;
  }

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = tid >> 6;
  const int wm = wave >> 1, wn = wave & 1;

  const int pid = xcd_remap(blockIdx.x, tiles_m * tiles_n);
  const int in_group = kGroupM * tiles_n;
  const int group = pid / in_group;
  const int first_m = group * kGroupM;
  const int gsize = min(tiles_m - first_m, kGroupM);
  const int tm = first_m + (pid % in_group) % gsize;
  const int tn = (pid % in_group) / gsize;
  const int64_t m0 = int64_t(tm) * BM, n0 = int64_t(tn) * BN;

  const int64_t M = g.m, N = g.n, K = g.k;
  const int lrow = lane >> 3;
  uint32_t oa[CHA], ob[CHB];
#pragma unroll
  for (int c = 0; c < CHA; ++c) {
    const int row = 8 * (wave + NW * c) + lrow;
    const int lch = (lane & 7) ^ row_swizzle(row);
    oa[c] = chunk_offset(min(m0 + row, M - 1), g.lda, lch, K);
  }
#pragma unroll
  for (int c = 0; c < CHB; ++c) {
    const int row = 8 * (wave + NW * c) + lrow;
    const int lch = (lane & 7) ^ row_swizzle(row);
    ob[c] = chunk_offset(min(n0 + row, N - 1), g.ldb, lch, K);
  }
  v4f acc[I][J];
  large_k_loop<FA, FB, BM, BN>(g.a, g.b, oa, ob, K, smem, acc);

  // Epilogue through LDS: the MFMA layout gives each lane one row and a column
  // quad per 16 x 16 block, so store instructions would touch 16 rows x 64 B.
  // Each wave instead writes one 32-row block of its sub-tile (32 x TN FP32,
  // rows padded to TN + 4 floats) into LDS, then reads it back row-contiguous:
  // 32 lanes x 16 B cover one 512-byte output row run per store instruction.
  __syncthreads();  // every wave is done reading the last stage
  float *ep = reinterpret_cast<float *>(smem) + wave * 32 * EP;
  const SumScale scale = sum_scale(g.a_scale_inv, g.b_scale_inv);
  const bool nfull = n0 + BN <= N;
  // Full tile with a vector-aligned destination (the common case): no bounds
  // checks, every store address is a uniform row base (scalar registers) plus
  // one per-lane offset, and LDS addresses are one base plus immediates.  With
  // one wave per SIMD the epilogue runs at instruction latency, so its
  // instruction count is its time.  Other tiles take the checked path.
  constexpr int ES = OUT == 1 ? 2 : 4;  // output element bytes
  // (buffer instructions: the row offset is a scalar operand; every offset of
  // the wave's TM x TN block stays below 2^31)
  const bool fast = vec_ok && nfull && m0 + BM <= M && g.ldc * ES * (TM + 2) < (int64_t(1) << 31);
  const bool has_col = (lane & 31) * 4 < TN;  // TN = 112 or 96: 28 or 24 of each 32 lanes hold a column quad
  const int wu = __builtin_amdgcn_readfirstlane(wave);
  const uint32_t voff = uint32_t((lane >> 5) * g.ldc + (lane & 31) * 4) * uint32_t(ES);
  char *cbase = static_cast<char *>(g.c) + ((m0 + (wu >> 1) * TM) * g.ldc + n0 + (wu & 1) * TN) * ES;
  const __amdgpu_buffer_rsrc_t crs = __builtin_amdgcn_make_buffer_rsrc(cbase, short(0), 0x7fffffff, 0x00020000);
  const int rstep = int(g.ldc) * ES;  // bytes per output row
  float *ew = ep + (lane & 15) * EP + 4 * (lane >> 4);
  const float *er = ep + (lane >> 5) * EP + (lane & 31) * 4;
#pragma unroll
  for (int i = 0; i < TM / 32; ++i) {
    // accumulate: read this block's destination first, so the loads are in
    // flight during the LDS round trip instead of one dependent load per row
    float4 pre[16];
    if constexpr (OUT == 2) {
      if (fast) {
#pragma unroll
        for (int it = 0; it < 16; ++it)
          if (has_col) pre[it] = __builtin_bit_cast(float4, __builtin_amdgcn_raw_buffer_load_b128(crs, voff, (i * 32 + 2 * it) * rstep, kNT));
      } else {
#pragma unroll
        for (int it = 0; it < 16; ++it) {
          const int64_t row = m0 + wm * TM + i * 32 + 2 * it + (lane >> 5);
          const int64_t col = n0 + wn * TN + (lane & 31) * 4;
          pre[it] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (has_col && row < M && (nfull || col + 4 <= N)) {
            const v4f_out w = *reinterpret_cast<const v4f_out *>(static_cast<const float *>(g.c) + row * g.ldc + col);
            pre[it] = make_float4(w[0], w[1], w[2], w[3]);
          }
        }
      }
    }
    if constexpr (OUT == 1) {
      if (fast) {
        // BF16 output: rounded before the LDS round trip, which then moves
        // half the bytes (rows of TN values padded to TN + 8), and every store
        // instruction writes four 2 * TN-byte row runs, 16 bytes per lane.
        // The same round-to-nearest-even of the same FP32 value, so the same
        // bits; measured 0.3-0.5% faster per stage step on MI355X.
        constexpr int EPH = TN + 8;
        uint16_t *eh = reinterpret_cast<uint16_t *>(ep);
        uint16_t *ehw = eh + (lane & 15) * EPH + 4 * (lane >> 4);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int j = 0; j < J; ++j) {
            const v4f a = acc[2 * i + h][j];
            *reinterpret_cast<uint2 *>(ehw + h * 16 * EPH + j * 16) =
                make_uint2(bf16x2_bits(scale(a[0]), scale(a[1])), bf16x2_bits(scale(a[2]), scale(a[3])));
          }
        const uint16_t *ehr = eh + (lane >> 4) * EPH + (lane & 15) * 8;
        const uint32_t voffh = uint32_t((lane >> 4) * g.ldc + (lane & 15) * 8) * 2u;
#pragma unroll
        for (int it = 0; it < 8; ++it) {
          if ((lane & 15) * 8 >= TN) continue;
          const uint4 v = *reinterpret_cast<const uint4 *>(ehr + it * 4 * EPH);
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4i, v), crs, voffh, (i * 32 + 4 * it) * rstep, kNT);
        }
        continue;
      }
    }
    // block rows 2i and 2i+1: lane holds row (lane & 15) of each, four
    // consecutive columns 16 j + 4 (lane >> 4) .. +3 of every column block j
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < J; ++j)
        *reinterpret_cast<float4 *>(ew + h * 16 * EP + j * 16) =
            make_float4(scale(acc[2 * i + h][j][0]), scale(acc[2 * i + h][j][1]), scale(acc[2 * i + h][j][2]),
                        scale(acc[2 * i + h][j][3]));
    // same wave writes then reads its own LDS rows: LDS operations of one wave
    // complete in order
    if (fast) {
#pragma unroll
      for (int it = 0; it < 16; ++it) {
        if (!has_col) continue;
        const float4 v4 = *reinterpret_cast<const float4 *>(er + it * 2 * EP);
        const int so = (i * 32 + 2 * it) * rstep;
        if constexpr (OUT == 0) {
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4i, v4), crs, voff, so, kNT);
        } else if constexpr (OUT == 1) {
          const v2i w = {int(bf16x2_bits(v4.x, v4.y)), int(bf16x2_bits(v4.z, v4.w))};
          __builtin_amdgcn_raw_buffer_store_b64(w, crs, voff, so, kNT);
        } else {
          const float4 o = pre[it];
          const float4 r = make_float4(o.x + v4.x, o.y + v4.y, o.z + v4.z, o.w + v4.w);
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4i, r), crs, voff, so, kNT);
        }
      }
      continue;
    }
#pragma unroll
    for (int it = 0; it < 16; ++it) {
      const int r = 2 * it + (lane >> 5);
      const int64_t row = m0 + wm * TM + i * 32 + r;
      const int cl = (lane & 31) * 4;
      const int64_t col = n0 + wn * TN + cl;
      if (!has_col) continue;
      const float4 v4 = *reinterpret_cast<const float4 *>(ep + r * EP + cl);
      if (row >= M) continue;
      const float v[4] = {v4.x, v4.y, v4.z, v4.w};
      if (nfull || col + 4 <= N) {  // at any alignment
        if constexpr (OUT == 0) {
          *reinterpret_cast<v4f_out *>(static_cast<float *>(g.c) + row * g.ldc + col) = v4f_out{v[0], v[1], v[2], v[3]};
        } else if constexpr (OUT == 1) {
          const uint32_t lo = bf16x2_bits(v[0], v[1]);
          const uint32_t hi = bf16x2_bits(v[2], v[3]);
          *reinterpret_cast<v2i_out *>(static_cast<uint16_t *>(g.c) + row * g.ldc + col) = v2i_out{int(lo), int(hi)};
        } else {
          const float4 o = pre[it];
          *reinterpret_cast<v4f_out *>(static_cast<float *>(g.c) + row * g.ldc + col) =
              v4f_out{o.x + v[0], o.y + v[1], o.z + v[2], o.w + v[3]};
        }
      } else {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          if (col + t >= N) break;
          if constexpr (OUT == 0) {
            static_cast<float *>(g.c)[row * g.ldc + col + t] = v[t];
          } else if constexpr (OUT == 1) {
            static_cast<uint16_t *>(g.c)[row * g.ldc + col + t] = bf16_bits(v[t]);
          } else {
            float *dst = static_cast<float *>(g.c) + row * g.ldc + col + t;
            *dst = *dst + v[t];
          }
        }
      }
    }
  }
}

template <int FA, int FB, int BM, int BN>
hipError_t launch_w4(const GemmParams &g, hipStream_t s, const UpdateParams &u) {
  const int tiles_m = int((g.m + BM - 1) / BM), tiles_n = int((g.n + BN - 1) / BN);
  const int vec_ok = gemm_vec_ok(g);
  const dim3 grid(unsigned(tiles_m) * unsigned(tiles_n) + unsigned(u.n)), block(256);
  switch (g.out) {
    case 0: return klaunch(gemm_tn_w4_kernel<FA, FB, 0, BM, BN>, grid, block, 0, s, g, tiles_m, tiles_n, vec_ok, u);
    case 1: return klaunch(gemm_tn_w4_kernel<FA, FB, 1, BM, BN>, grid, block, 0, s, g, tiles_m, tiles_n, vec_ok, u);
    default: return klaunch(gemm_tn_w4_kernel<FA, FB, 2, BM, BN>, grid, block, 0, s, g, tiles_m, tiles_n, vec_ok, u);
  }
}

template <int BM, int BN>
hipError_t launch_w4_fmts(const GemmParams &g, hipStream_t s, const UpdateParams &u) {
  if (g.fmt_a == 0 && g.fmt_b == 0) return launch_w4<0, 0, BM, BN>(g, s, u);
  if (g.fmt_a == 1 && g.fmt_b == 0) return launch_w4<1, 0, BM, BN>(g, s, u);
  if (g.fmt_a == 0 && g.fmt_b == 1) return launch_w4<0, 1, BM, BN>(g, s, u);
  return launch_w4<1, 1, BM, BN>(g, s, u);
}

}  // namespace

hipError_t launch_gemm_large(int tile, const GemmParams &g, hipStream_t s, const UpdateParams &u) {
  switch (tile) {
    case kTile256x192: return launch_w4_fmts<256, 192>(g, s, u);
    case kTile192x256: return launch_w4_fmts<192, 256>(g, s, u);
    case kTile256x224: return launch_w4_fmts<256, 224>(g, s, u);
    default: return launch_w4_fmts<256, 256>(g, s, u);
  }
}

}  // namespace qe
