// The K loops of the FP8 products (gfx950), shared by the plain GEMM
// (gemm_fp8.hip, gemm_ring.hip, where their schedules are described) and by the
// products with an epilogue of their own (act_gemm.hip).  Each adds a tile's
// whole reduction to zeroed accumulators.
//
// a, b: bases of the operands (uniform in the wave; they may differ from wave to
// wave); oa, ob: byte offsets of the lane's LDS-bound loads from them, chunk
// `(lane & 7) ^ row_swizzle(row)` of LDS row 8 (wave + 4 c) + lane / 8 for load c.
// On return some wave may still be reading the stages: a barrier comes before
// anything else is written there.
#pragma once

#include "gemm_util.h"

namespace qe {
namespace {

// Operands of one scale each: the sums are scaled after the loop.
struct NoScales {
  static constexpr bool kOn = false;
};

// Operands with a scale for each block of 128 along the reduction, one byte (the
// exponent field of a power of two) per row and K tile, which the matrix instruction
// applies to its products by itself: it takes a scale for 32 values of a row, the four
// of a K tile are the same.  The bytes come four K tiles (a group) at a time, a word
// of every tile row by an LDS-bound load, and go through BUFS buffers of the groups
// modulo BUFS at byte `lds` of smem: those of A's rows, then of B's.  A fragment's
// word stays in a register for the group's four tiles, and the instruction selects
// the byte.  Against a group's other traffic that is two LDS-bound loads in 64 of a
// wave and 16 word reads in 128 of fragments (256 x 256 tiles).
template <int BM, int BN, int BUFS>
struct LdsScales {
  static constexpr bool kOn = true;
  static constexpr int kSlots = (BM + BN) / 64, kPer = (kSlots + 3) / 4;  // 64 rows each; per wave
  static constexpr int kBuf = (BM + BN) * 4, kBytes = BUFS * kBuf;
  static_assert((BUFS & (BUFS - 1)) == 0, "buffers are numbered by bits");
  const uint8_t *base[kPer];  // uniform in the wave
  uint32_t off[kPer];
  int groups;
  uint32_t lds;
  __device__ __forceinline__ void load(const uint8_t *smem, int wave, int group) const {
    if (group >= groups) return;
    const uint32_t to = uint32_t(reinterpret_cast<uintptr_t>(smem)) + lds + uint32_t(group & (BUFS - 1)) * kBuf;
#pragma unroll
    for (int q = 0; q < kPer; ++q) {
      const int slot = __builtin_amdgcn_readfirstlane(wave + 4 * q);
      if (slot < kSlots)
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(off[q]), "s"(base[q] + 4 * group),
                     "s"(__builtin_amdgcn_readfirstlane(to + uint32_t(slot) * 256u)) : "memory", "m0");
    }
  }
  // Where the words of rows `row` .. of a group start; the compiler sees an address and
  // constants from it, not the parts of it that it would keep one register each for.
  __device__ __forceinline__ uint32_t at(const uint8_t *smem, int row, int group) const {
    uint32_t p = uint32_t(reinterpret_cast<uintptr_t>(smem)) + lds + uint32_t(group & (BUFS - 1)) * kBuf + uint32_t(row) * 4u;
    asm("" : "+v"(p));
    return p;
  }
  static __device__ __forceinline__ int read(uint32_t p, int rows) {
    return *reinterpret_cast<const __attribute__((address_space(3))) int *>(p + uint32_t(rows) * 4u);
  }
  static __device__ __forceinline__ int read_byte(uint32_t p, int rows) {
    return *reinterpret_cast<const __attribute__((address_space(3))) uint8_t *>(p + uint32_t(rows) * 4u);
  }
};

// One block's product of a K tile.  With scales it is inline assembly, because the
// compiler gives the builtin's result registers of its own, apart from the
// accumulator's (the 256 x 256 tile then spills 80 registers and the 128 x 128 one
// 140).  The assembler adds no waits: s_nop 1 stands for what a vector instruction
// that wrote an operand needs, products of the same accumulator are at least three
// others apart in the loops, and settle() comes before anything else reads them.
// Nothing here keeps the compiler from copying a sum in between: tests/test_mfma_waits.py
// follows the built kernels' paths and finds an instruction that touches one too early.
// BYTE: which byte of sa, sb is the K tile's.
#define QE_MFMA_SCALED(SEL)                                                                                       \
  asm volatile("s_nop 1\n\tv_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 " SEL " cbsz:%5 blgp:%6"       \
               : "+a"(acc) : "v"(b), "v"(a), "v"(sb), "v"(sa), "n"(FB), "n"(FA))
template <int FA, int FB, bool SCALED, int BYTE>
__device__ __forceinline__ void mfma_tile(v4f &acc, const v8i &a, const v8i &b, int sa, int sb) {
  if constexpr (!SCALED)
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, acc, FB, FA, 0, 0, 0, 0);
  else if constexpr (BYTE == 0)
    QE_MFMA_SCALED("op_sel_hi:[0,0,0]");
  else if constexpr (BYTE == 1)
    QE_MFMA_SCALED("op_sel:[1,1,0] op_sel_hi:[0,0,0]");
  else if constexpr (BYTE == 2)
    QE_MFMA_SCALED("op_sel_hi:[1,1,0]");
  else
    QE_MFMA_SCALED("op_sel:[1,1,0] op_sel_hi:[1,1,0]");
}
#undef QE_MFMA_SCALED
// After the last of them: longer than the instruction takes to write its result (12 wait states).
template <bool SCALED, int I, int J>
__device__ __forceinline__ void settle(v4f (&acc)[I][J]) {
  if constexpr (SCALED) {
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
      for (int j = 0; j < J; ++j) asm volatile("" : "+a"(acc[i][j]));
  }
}

// Large tiles, four waves, two K stages in smem (and one 1 KB block per wave):
// see gemm_tn_w4_kernel.  The offsets come from chunk_offset.
template <int FA, int FB, int BM, int BN, typename SC = NoScales>
__device__ __forceinline__ void large_k_loop(const uint8_t *a, const uint8_t *b, const uint32_t (&oa)[BM / 32],
                                             const uint32_t (&ob)[BN / 32], int64_t K, uint8_t *smem,
                                             v4f (&acc)[BM / 32][BN / 32], const SC &sc = SC{}) {
  constexpr int NW = 4, TM = BM / 2, TN = BN / 2;
  constexpr int I = TM / 16, J = TN / 16;    // 16 x 16 MFMA blocks per wave sub-tile
  constexpr int IA = I / 2, IB = I - IA;     // block rows of phase A and phase B
  constexpr int QA = IA * J, QB = IB * J;    // MFMAs per phase
  constexpr int CHA = BM / 32, CHB = BN / 32;  // 16-byte LDS-bound loads per lane per K tile
  constexpr int ND = CHA + CHB;              // LDS-bound loads per K tile
  constexpr int STAGE = (BM + BN) * BK;
  static_assert(CHA * NW * 1024 == BM * BK, "LDS-bound load d of a tile lands at stage + 4096 d");
  const int lane = threadIdx.x & 63;
  const int wave = SC::kOn ? __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6) : int(threadIdx.x) >> 6;
  const int wm = wave >> 1, wn = wave & 1;
  const int lrow = lane >> 3;
  const int KT = int(K / BK);
  const int64_t ktail = K - int64_t(KT) * BK;
  const int T = KT + (ktail > 0 ? 1 : 0);

  const uint32_t lds_base = uint32_t(reinterpret_cast<uintptr_t>(smem));
  const uint32_t wblk = __builtin_amdgcn_readfirstlane(lds_base + uint32_t(wave) * 1024u);
  const uint32_t wdummy = __builtin_amdgcn_readfirstlane(lds_base + uint32_t(2 * STAGE) + uint32_t(wave) * 1024u);

  // The 64-bit form of an offset, which only the partial K tile needs, is made there
  // (the compiler keeps it through the loop otherwise: 16 registers that the scales take).
  auto here = [](uint32_t o) {
    if constexpr (SC::kOn) asm volatile("" : "+v"(o));
    return o;
  };
  auto issue = [&](int kt, int buf) {
    if (kt < KT) {
      const uint8_t *ga = a + int64_t(kt) * BK;
      const uint8_t *gb = b + int64_t(kt) * BK;
      const uint32_t sa = wblk + uint32_t(buf * STAGE);
      const uint32_t sb = sa + uint32_t(BM * BK);
#pragma unroll
      for (int c = 0; c < CHA; ++c)
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(oa[c]), "s"(ga),
                     "s"(sa + uint32_t(c * NW * 1024)) : "memory", "m0");
#pragma unroll
      for (int c = 0; c < CHB; ++c)
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(ob[c]), "s"(gb),
                     "s"(sb + uint32_t(c * NW * 1024)) : "memory", "m0");
    } else {  // the last, partial K tile, through registers: bytes at or past K are zero
      uint8_t *dA = smem + buf * STAGE;
      uint8_t *dB = dA + BM * BK;
      const uint32_t k0 = uint32_t(KT) * BK;
#pragma unroll
      for (int c = 0; c < CHA; ++c) {
        const int row = 8 * (wave + NW * c) + lrow;
        const int64_t gk = int64_t(k0) + ((lane & 7) ^ row_swizzle(row)) * 16;
        const uint4 va = gk < K ? mask_tail(*reinterpret_cast<const uint4 *>(a + (here(oa[c]) + k0)), K - gk) : make_uint4(0u, 0u, 0u, 0u);
        *reinterpret_cast<uint4 *>(dA + (wave + NW * c) * 1024 + lane * 16) = va;
      }
#pragma unroll
      for (int c = 0; c < CHB; ++c) {
        const int row = 8 * (wave + NW * c) + lrow;
        const int64_t gk = int64_t(k0) + ((lane & 7) ^ row_swizzle(row)) * 16;
        const uint4 vb = gk < K ? mask_tail(*reinterpret_cast<const uint4 *>(b + (here(ob[c]) + k0)), K - gk) : make_uint4(0u, 0u, 0u, 0u);
        *reinterpret_cast<uint4 *>(dB + (wave + NW * c) * 1024 + lane * 16) = vb;
      }
    }
  };

  // 16-row fragments: lane l reads row (l & 15), the 32 bytes 32 (l >> 4) .. +31
  // of the K tile, i.e. logical chunks 2 (l >> 4) and the next.  The swizzle
  // term depends on (l & 15) only, so every fragment is base + constant.
  const int fr = lane & 15, fq = lane >> 4;
  const uint32_t f_lo = uint32_t(fr) * BK + uint32_t((2 * fq) ^ row_swizzle(fr)) * 16;
  const uint32_t f_hi = uint32_t(fr) * BK + uint32_t((2 * fq + 1) ^ row_swizzle(fr)) * 16;
  auto frag = [&](const uint8_t *base) -> v8i {
    const uint4 lo = *reinterpret_cast<const uint4 *>(base + f_lo);
    const uint4 hi = *reinterpret_cast<const uint4 *>(base + f_hi);
    return v8i{int(lo.x), int(lo.y), int(lo.z), int(lo.w), int(hi.x), int(hi.y), int(hi.z), int(hi.w)};
  };
  int sa[I], sb[J];  // the fragments' scales, read with them from pa, pb
  uint32_t pa = 0, pb = 0;
  auto scales_at = [&](int group) {
    if constexpr (SC::kOn) {
      pa = sc.at(smem, wm * TM + fr, group);
      pb = sc.at(smem, BM + wn * TN + fr, group);
    }
  };
  // `byte`: that of the tile, t % 4; the group's words come with its first tile.
  auto read_a = [&](auto byte, int buf, int i, v8i (&fa)[I]) {
    fa[i] = frag(smem + buf * STAGE + (wm * TM + i * 16) * BK);
    if constexpr (SC::kOn) {
      if constexpr (decltype(byte)::value == 0) sa[i] = SC::read(pa, i * 16);
    }
  };
  auto read_b = [&](auto byte, int buf, int j, v8i (&fb)[J]) {
    fb[j] = frag(smem + buf * STAGE + (BM + wn * TN + j * 16) * BK);
    if constexpr (SC::kOn) {
      if constexpr (decltype(byte)::value == 0) sb[j] = SC::read(pb, j * 16);
    }
  };

#pragma unroll
  for (int i = 0; i < I; ++i)
#pragma unroll
    for (int j = 0; j < J; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};

  auto mfma = [&](auto byte, int i, int j, const v8i (&fa)[I], const v8i (&fb)[J]) {
    mfma_tile<FA, FB, SC::kOn, decltype(byte)::value>(acc[i][j], fa[i], fb[j], sa[i], sb[j]);
  };
  // LDS-bound loads inside the K loop, two instructions each: load d of a K
  // tile lands at stage + 4096 d, so M0 steps by a uniform stride, and the
  // step is issued before an MFMA and the load after it (the MFMA is the wait
  // state M0 needs).  Past the last full K tile the loads still run, from
  // tile 0 into the wave's dummy block with stride 0: no branch per load (and
  // no byte past a row of less than 128, see chunk_offset).
  auto dma_m0 = [&](int d, uint32_t base, uint32_t stride) {
    if (d == 0)
      asm volatile("s_mov_b32 m0, %0" ::"s"(base) : "m0");
    else
      asm volatile("s_add_u32 m0, m0, %0" ::"s"(stride) : "m0", "scc");
  };
  auto dma_load = [&](int d, const uint8_t *ga, const uint8_t *gb) {
    if (d < CHA)
      asm volatile("global_load_lds_dwordx4 %0, %1" ::"v"(oa[d]), "s"(ga) : "memory");
    else
      asm volatile("global_load_lds_dwordx4 %0, %1" ::"v"(ob[d - CHA]), "s"(gb) : "memory");
  };

  // Phase A of a tile from stage `buf`: column-major MFMAs over block rows
  // 0 .. IA-1 (B fragment j is first needed at MFMA j * IA, so the fragments
  // read last in the previous phase B are needed last); A fragments IA .. I-1
  // of the same tile are read after the first MFMAs (one per even slot), long
  // before phase B needs them.  The tile's B fragments are all in registers
  // by now, so the same stage's B half already takes the B part of the tile
  // two K tiles ahead (`kt3`), spread over the phase: a K step and a half
  // before it is read.
  auto b_slot = [](int q, int k) { return (k * QA) / CHB + 1 == q; };
  auto phase_a = [&](auto byte, int buf, bool dmab, int kt3, v8i (&fa)[I], v8i (&fb)[J]) {
    const uint8_t *gb = dmab ? b + int64_t(kt3) * BK : b;
    const uint32_t base = dmab ? wblk + uint32_t(buf * STAGE + BM * BK) : wdummy;
    const uint32_t stride = dmab ? uint32_t(NW * 1024) : 0u;
#pragma unroll
    for (int q = 0; q < QA; ++q) {
      int d = -1;  // the B-part load of this slot (folds to a constant once unrolled)
#pragma unroll
      for (int k = 0; k < CHB; ++k) d = b_slot(q, k) ? k : d;
      __builtin_amdgcn_sched_barrier(0);
      if (d >= 0) dma_m0(d, base, stride);
      __builtin_amdgcn_sched_barrier(0);
      mfma(byte, q % IA, q / IA, fa, fb);
      __builtin_amdgcn_sched_barrier(0);
      if (d >= 0) dma_load(CHA + d, a, gb);
      if (q % 2 == 0 && q / 2 < IB) read_a(byte, buf, IA + q / 2, fa);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  // Phase B of a tile: column-major MFMAs over block rows IA .. I-1.  After
  // the last use of B fragment j, the next tile's B fragment j is read from
  // stage `nbuf` into the same registers; the next tile's A fragments
  // 0 .. IA-1 are read in the first slots (their registers are free since
  // phase A).  `dma` issues the A part of tile `kt2` into stage `buf`.
  // Slots of phase B, one kind of memory instruction each where possible: the
  // next tile's A fragments after MFMAs 0, 4, 8, ..; LDS-bound loads after
  // MFMAs q = 1, 2 (mod 4), so the A part is issued in the first half of the
  // phase; B fragments after the last use of each (q = 3 (mod 4) when IB =
  // 4).  Loads that do not fit go to the latest q = 0 (mod 4) slots past the A
  // reads.  (Measured: the A part spread over all of phase B instead, equal;
  // the B part packed into the first half of phase A, 0.5% slower.)
  auto load_slot = [](int q) -> bool {
    constexpr int n12 = (QB / 4) * 2;
    if (q % 4 == 1 || q % 4 == 2) return (q / 4) * 2 + (q % 4 - 1) < CHA;
    if (q % 4 == 0 && CHA > n12) return q / 4 >= IA && QB / 4 - 1 - q / 4 < CHA - n12;
    return false;
  };
  auto phase_b = [&](auto byte, int nbuf, bool dma, int kt2, int buf, v8i (&fa)[I], v8i (&fb)[J]) {
    static_assert(QB % 4 == 0, "phase B slots come in fours");
    constexpr std::integral_constant<int, (decltype(byte)::value + 1) % 4> next{};
    const uint8_t *ga = dma ? a + int64_t(kt2) * BK : a;
    const uint8_t *gb = dma ? b + int64_t(kt2) * BK : b;
    const uint32_t base = dma ? wblk + uint32_t(buf * STAGE) : wdummy;
    const uint32_t stride = dma ? uint32_t(NW * 1024) : 0u;
#pragma unroll
    for (int q = 0; q < QB; ++q) {
      const int j = q / IB, i = IA + q % IB;
      const bool ld = load_slot(q);
      int d = 0;  // loads in earlier slots (folds to a constant once unrolled)
#pragma unroll
      for (int r = 0; r < q; ++r) d += load_slot(r) ? 1 : 0;
      __builtin_amdgcn_sched_barrier(0);
      if (ld) dma_m0(d, base, stride);
      __builtin_amdgcn_sched_barrier(0);  // M0 is written before the MFMA, never next to the load
      mfma(byte, i, j, fa, fb);
      __builtin_amdgcn_sched_barrier(0);
      if (ld) dma_load(d, ga, gb);
      if (q % 4 == 0 && q / 4 < IA) read_a(next, nbuf, q / 4, fa);
      if (q % IB == IB - 1) read_b(next, nbuf, j, fb);  // last use of B fragment j was this MFMA
    }
    __builtin_amdgcn_sched_barrier(0);
  };

  if (T > 0) {
    v8i fa[I], fb[J];
    constexpr std::integral_constant<int, 0> first{};
    if constexpr (SC::kOn) sc.load(smem, wave, 0);  // the first loads: complete whenever a tile's are
    issue(0, 0);
    if (KT > 1) {
      // both first K tiles are full: tile 1's LDS-bound loads stay in flight
      // while the wave waits for its tile-0 loads (the ND most recent ones
      // are tile 1's; the counter completes in order)
      issue(1, 1);
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(ND) : "memory");
    } else {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    __syncthreads();
    scales_at(0);
#pragma unroll
    for (int j = 0; j < J; ++j) read_b(first, 0, j, fb);
#pragma unroll
    for (int i = 0; i < IA; ++i) read_a(first, 0, i, fa);
    if (T > 1 && KT <= 1) issue(1, 1);  // tile 1 is the partial tail: through registers
    __syncthreads();                       // every wave holds tile 0's B fragments: stage 0's B half is free
    phase_a(first, 0, 2 < KT, 2, fa, fb);         // and takes tile 2's B part
    // tile 1 complete; the CHB most recent loads (tile 2's B part) may still
    // be in flight: the counter completes in order
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(CHB) : "memory");
    __syncthreads();                       // tile 1 published; tile 0 fully read
    if constexpr (SC::kOn) {  // four tiles a turn: which byte is part of the instruction
      auto step = [&](int t, int buf, auto byte) {  // as below
        constexpr std::integral_constant<int, (decltype(byte)::value + 1) % 4> next{};
        const bool dma = t + 2 < KT;
        if (t + 2 < T && !dma) issue(t + 2, buf);
        // The next group's scales, into the buffer whose last reads were of tile t - 1.
        // They are older than the B part below, so the wait at this step's end covers
        // them: three steps before they are read.
        if constexpr (decltype(byte)::value == 0) sc.load(smem, wave, t / 4 + 1);
        if constexpr (decltype(next)::value == 0) scales_at(t / 4 + 1);
        phase_b(byte, buf ^ 1, dma, t + 2, buf, fa, fb);
        if (t + 1 < T) {
          __syncthreads();
          phase_a(next, buf ^ 1, t + 3 < KT, t + 3, fa, fb);
          asm volatile("s_waitcnt vmcnt(%0)" ::"n"(CHB) : "memory");
          __syncthreads();
        }
      };
      for (int t = 0; t < T; t += 4) {
        step(t, 0, first);
        if (t + 1 < T) step(t + 1, 1, std::integral_constant<int, 1>{});
        if (t + 2 < T) step(t + 2, 0, std::integral_constant<int, 2>{});
        if (t + 3 < T) step(t + 3, 1, std::integral_constant<int, 3>{});
      }
    } else {  // (through step the loop has three more branches a tile: 1% on large products)
      for (int t = 0; t < T; ++t) {
        const int buf = t & 1;
        const bool dma = t + 2 < KT;
        if (t + 2 < T && !dma) issue(t + 2, buf);
        // phase B of tile t, with tile t+2's A part; reads of tile t+1 (in the
        // last iteration they read a stale stage that is never used: always in
        // bounds, and branch-free here)
        phase_b(first, buf ^ 1, dma, t + 2, buf, fa, fb);
        if (t + 1 < T) {
          __syncthreads();                   // tile t+1's B fragments read by every wave
          phase_a(first, buf ^ 1, t + 3 < KT, t + 3, fa, fb);  // with tile t+3's B part
          asm volatile("s_waitcnt vmcnt(%0)" ::"n"(CHB) : "memory");
          __syncthreads();                   // tile t+2 published; tile t+1 fully read
        }
      }
    }
    settle<SC::kOn>(acc);
  }
}

// Bytes [0, valid) of a 32-byte fragment kept, the rest zeroed.
__device__ __forceinline__ v8i mask_frag(v8i f, int valid) {
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    const int nb = valid - 4 * q;
    const int k = nb <= 0 ? 0 : (nb >= 4 ? 4 : nb);
    f[q] &= int(uint32_t((uint64_t(1) << (8 * k)) - 1u));
  }
  return f;
}

// Ring tiles, four waves, S K stages in smem: see gemm_tn_ring_kernel.
template <int FA, int FB, int BM, int BN, int S, typename SC = NoScales>
__device__ __forceinline__ void ring_k_loop(const uint8_t *a, const uint8_t *b, const uint32_t (&oa)[BM / 32],
                                            const uint32_t (&ob)[BN / 32], int K, uint8_t *smem,
                                            v4f (&acc)[BM / 32][BN / 32], const SC &sc = SC{}) {
  constexpr int NW = 4, TM = BM / 2, TN = BN / 2;
  constexpr int I = TM / 16, J = TN / 16;
  constexpr int CHA = BM / 32, CHB = BN / 32;  // LDS-bound loads per lane per K tile
  constexpr int L = CHA + CHB;
  constexpr int Q = I * J;                     // MFMAs per wave and K tile
  constexpr int STAGE = (BM + BN) * BK;
  static_assert((S - 1) * L < 64, "the load counter holds 63");
  const int lane = threadIdx.x & 63;
  const int wave = SC::kOn ? __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6) : int(threadIdx.x) >> 6;
  const int wm = wave >> 1, wn = wave & 1;
  const int lrow = lane >> 3;
  const int ktail = K % BK;
  const int T = K / BK + (ktail > 0 ? 1 : 0);

  const uint32_t lds_base = uint32_t(reinterpret_cast<uintptr_t>(smem));
  const uint32_t wblk = __builtin_amdgcn_readfirstlane(lds_base + uint32_t(wave) * 1024u);

  auto load16 = [](uint32_t off, const uint8_t *base, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(lds)
                 : "memory", "m0");
  };
  auto issue = [&](int t, uint32_t stage) {
    const uint8_t *ga = a + int64_t(t) * BK;
    const uint8_t *gb = b + int64_t(t) * BK;
    const uint32_t sa = wblk + stage, sb = sa + uint32_t(BM * BK);
    if (ktail == 0 || t + 1 < T) {
#pragma unroll
      for (int c = 0; c < CHA; ++c) load16(oa[c], ga, sa + uint32_t(c * NW * 1024));
#pragma unroll
      for (int c = 0; c < CHB; ++c) load16(ob[c], gb, sb + uint32_t(c * NW * 1024));
    } else {  // chunks past the row's last 16 bytes re-read its last chunk; the fragments mask them
      const int last = (ktail - 1) >> 4;
#pragma unroll
      for (int c = 0; c < CHA; ++c) {
        const int row = 8 * (wave + NW * c) + lrow;
        const int ch = (lane & 7) ^ row_swizzle(row);
        load16(oa[c] - uint32_t(max(ch - last, 0) * 16), ga, sa + uint32_t(c * NW * 1024));
      }
#pragma unroll
      for (int c = 0; c < CHB; ++c) {
        const int row = 8 * (wave + NW * c) + lrow;
        const int ch = (lane & 7) ^ row_swizzle(row);
        load16(ob[c] - uint32_t(max(ch - last, 0) * 16), gb, sb + uint32_t(c * NW * 1024));
      }
    }
  };

  // 16-row fragments: lane l holds row (l & 15), bytes 32 (l >> 4) .. +31 of
  // the K tile (the layout of the large tiles).
  const int fr = lane & 15, fq = lane >> 4;
  const uint32_t f_lo = uint32_t(fr) * BK + uint32_t((2 * fq) ^ row_swizzle(fr)) * 16;
  const uint32_t f_hi = uint32_t(fr) * BK + uint32_t((2 * fq + 1) ^ row_swizzle(fr)) * 16;
  auto frag = [&](uint32_t base) -> v8i {
    const uint4 lo = *reinterpret_cast<const uint4 *>(smem + base + f_lo);
    const uint4 hi = *reinterpret_cast<const uint4 *>(smem + base + f_hi);
    return v8i{int(lo.x), int(lo.y), int(lo.z), int(lo.w), int(hi.x), int(hi.y), int(hi.z), int(hi.w)};
  };
  struct Frags {
    v8i a[I], b[J];
    int sa[I], sb[J];  // their scales
  };
  uint32_t pa = 0, pb = 0;  // where the scales of the tile that is read start
  auto scales_at = [&](int t) {
    if constexpr (SC::kOn) {
      pa = sc.at(smem, wm * TM + fr, t / 4) + uint32_t(t % 4);
      pb = sc.at(smem, BM + wn * TN + fr, t / 4) + uint32_t(t % 4);
    }
  };
  auto read_a = [&](uint32_t stage, int i, Frags &f) {
    f.a[i] = frag(stage + uint32_t((wm * TM + i * 16) * BK));
    if constexpr (SC::kOn) f.sa[i] = SC::read_byte(pa, i * 16);
  };
  auto read_b = [&](uint32_t stage, int j, Frags &f) {
    f.b[j] = frag(stage + uint32_t((BM + wn * TN + j * 16) * BK));
    if constexpr (SC::kOn) f.sb[j] = SC::read_byte(pb, j * 16);
  };
  auto read = [&](int t, uint32_t stage, Frags &f) {
    scales_at(t);
#pragma unroll
    for (int i = 0; i < I; ++i) read_a(stage, i, f);
#pragma unroll
    for (int j = 0; j < J; ++j) read_b(stage, j, f);
  };
  // Scales go two groups ahead: at least seven tiles' loads are younger than theirs
  // when they are read, more than the waits leave in flight.
  static_assert(S - 2 <= 7, "a group's scales are complete when they are read");
  auto load_scales = [&](int t) {
    if constexpr (SC::kOn)
      if ((t & 3) == 0) sc.load(smem, wave, (t >> 2) + 2);
  };
  auto mask = [&](Frags &f) {
    const int valid = ktail - 32 * fq;
#pragma unroll
    for (int i = 0; i < I; ++i) f.a[i] = mask_frag(f.a[i], valid);
#pragma unroll
    for (int j = 0; j < J; ++j) f.b[j] = mask_frag(f.b[j], valid);
  };

#pragma unroll
  for (int i = 0; i < I; ++i)
#pragma unroll
    for (int j = 0; j < J; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};

  auto mfma = [&](int i, int j, const Frags &f) {
    mfma_tile<FA, FB, SC::kOn, 0>(acc[i][j], f.a[i], f.b[j], f.sa[i], f.sb[j]);
  };
  uint32_t rd = 0;  // stage of tile t
  // Step t: fragments of tile t are in `cur`; tile t + 1's are read into `nxt`.
  // main_step (tile t + S exists and is full): after each MFMA, in a fixed
  // order, one LDS-bound load and one fragment read where they are due, so the
  // three pipes (MFMA, LDS, address) work side by side in a single wave.
  auto main_step = [&](int t, const Frags &cur, Frags &nxt) {
    // tile t + 1 complete: of the tiles issued so far, t + 2 .. t + S - 1 may
    // still be in flight (the counter completes in order)
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((S - 2) * L) : "memory");
    __syncthreads();  // tile t + 1 published; every wave holds tile t's fragments
    const uint8_t *ga = a + int64_t(t + S) * BK;
    const uint8_t *gb = b + int64_t(t + S) * BK;
    const uint32_t sa = wblk + rd;  // tile t's stage takes tile t + S; load d lands at sa + 4096 d
    rd = rd + STAGE == uint32_t(S * STAGE) ? 0u : rd + STAGE;
    load_scales(t);
    scales_at(t + 1);
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int d = 0; d < L; ++d)
        if (d * Q / L == q) {
          if (d == 0)
            asm volatile("s_mov_b32 m0, %0" ::"s"(sa) : "m0");
          else
            asm volatile("s_add_u32 m0, m0, %0" ::"n"(NW * 1024) : "m0", "scc");
        }
      __builtin_amdgcn_sched_barrier(0);  // M0 is written before the MFMA, never next to the load
      mfma(q / J, q % J, cur);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int d = 0; d < L; ++d)
        if (d * Q / L == q) {
          if (d < CHA)
            asm volatile("global_load_lds_dwordx4 %0, %1" ::"v"(oa[d]), "s"(ga) : "memory");
          else
            asm volatile("global_load_lds_dwordx4 %0, %1" ::"v"(ob[d - CHA]), "s"(gb) : "memory");
        }
#pragma unroll
      for (int r = 0; r < I + J; ++r)
        if (r * Q / (I + J) == q) {
          if (r < I)
            read_a(rd, r, nxt);
          else
            read_b(rd, r - I, nxt);
        }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  // The last steps: no tile, or the partial one, left to issue.  (Past the last
  // tile a stale stage is read and never used, so that the reads stay
  // branch-free and the compiler can wait for them one by one.)
  auto last_step = [&](int t, const Frags &cur, Frags &nxt) {
    if (t + S <= T)
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"((S - 2) * L) : "memory");
    else
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    const uint32_t freed = rd;
    rd = rd + STAGE == uint32_t(S * STAGE) ? 0u : rd + STAGE;
    read(t + 1, rd, nxt);
    __builtin_amdgcn_sched_barrier(0);
    load_scales(t);
    if (t + S < T) issue(t + S, freed);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int q = 0; q < Q; ++q) mfma(q / J, q % J, cur);
    __builtin_amdgcn_sched_barrier(0);
    if (t + 2 == T && ktail != 0) mask(nxt);
  };

  if (T > 0) {
    Frags f0, f1;
    if constexpr (SC::kOn) {
      sc.load(smem, wave, 0);
      sc.load(smem, wave, 1);
    }
#pragma unroll
    for (int t = 0; t < S; ++t)
      if (t < T) issue(t, uint32_t(t * STAGE));
    if (T >= S)
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"((S - 1) * L) : "memory");
    else
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    read(0, 0, f0);
    if (T == 1 && ktail != 0) mask(f0);
    int t = 0;
    for (; t + 1 + S < K / BK; t += 2) {
      main_step(t, f0, f1);
      main_step(t + 1, f1, f0);
    }
    for (; t + 1 < T; t += 2) {
      last_step(t, f0, f1);
      last_step(t + 1, f1, f0);
    }
    if (t < T) {
#pragma unroll
      for (int q = 0; q < Q; ++q) mfma(q / J, q % J, f0);
    }
    settle<SC::kOn>(acc);
  }
}

}  // namespace
}  // namespace qe
