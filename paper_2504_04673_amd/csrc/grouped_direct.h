// The grouped products of bfloat16 tensors whose rows begin on 16 bytes: operands go from memory into LDS without
// passing through registers, several steps ahead of the matrix cores.
//
// Bound: the matrix cores where every weight meets a few hundred rows, the weights' traffic below that.  A workgroup owns 256 x 256 of
// the result, eight wavefronts of 128 x 64: LDS has to deliver (rows + columns) of a wavefront's tile for rows x columns of
// work, 96 bytes a cycle and CU at 128 x 64, 128 at 64 x 64.  Two wavefronts share a SIMD, so that one's products fill the
// other's waits.  Four steps of 32 are in flight, so that a load has three steps' arithmetic to arrive.
#pragma once
#include "grouped.h"

namespace sagnn {

// Steps of 32 of the summed index; kStages of them in LDS
constexpr int kStep = 32, kStages = 4;

// A wavefront's 64 lanes write 1024 bytes of LDS one behind the other, so the order inside a tile is made by the addresses
// that the lanes load from.  Sixteen bytes are a granule.
// Summed index inside (ROWS rows of 64 bytes a step): two steps are loaded together, 128 bytes of eight rows an instruction, since half a
// cache line at a time takes each line out of the L2 twice (8192^3, both operands so: 1230 us).  LDS has the eight rows' halves for the first step, then
// those for the second.  Granule g of a row's four lies at g ^ swizzle(row), which spreads the rows that a read takes at once
// over the banks.  TR ([32][ROWS]): pairs of granules, since a transposing read takes 32 bytes of a row.
__device__ __forceinline__ int row_swizzle(int r) { return (r >> 2) & 3; }
__device__ __forceinline__ int sum_swizzle(int k) { return (k & 3) * 2; }

// The tile of an operand: ROWS rows (columns), loaded `kUnit` steps at a time
template <bool TR, int ROWS, int WAVES>
struct DirectOperand {
  static constexpr int kUnit = TR ? 1 : 2;
  static constexpr int kStageBytes = ROWS * kStep * 2, kBytes = kStages * kStageBytes;
  static constexpr int kLoads = kUnit * kStageBytes / 1024 / WAVES;      // instructions a wavefront and unit
  static constexpr int kLanes = TR ? ROWS / 8 : 8;                       // lanes along a row of memory
  static_assert(kLoads * WAVES * 1024 == kUnit * kStageBytes, "a unit must be whole instructions of every wavefront");
  static_assert(TR || kLoads % 2 == 0, "the swizzle of a wavefront's instructions alternates");
  const char* base;      // corner of the next unit to be loaded
  int64_t step;          // bytes to the one after it
  int64_t left;          // bytes from the corner to the end of the operand's last row
  int sum;               // of the summed index, from the next unit on
  uint32_t at[kLoads];   // of this lane, from the corner
  int inner;             // first of its eight elements inside a row (every load's)

  __device__ __forceinline__ void init(const __bf16* corner, int64_t ld, int rows, int total, int lane, int wave) {
    base = reinterpret_cast<const char*>(corner);
    step = TR ? kStep * ld * 2 : kUnit * kStep * 2;
    left = ((int64_t)((TR ? total : rows) - 1) * ld + (TR ? rows : total)) * 2;
    sum = total;
    inner = 0;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int first = (wave * kLoads + j) * (64 / kLanes);
      const int outer = first + (TR ? lane / kLanes : (lane & 31) / 4);
      const int granule = TR ? (lane % kLanes) ^ (2 * sum_swizzle(outer) % kLanes) : (lane >> 5) * 4 + ((lane & 3) ^ row_swizzle(outer));
      at[j] = (uint32_t)(outer * ld * 2) + granule * 16;
      if (TR && granule * 8 >= rows) at[j] = 0x80000000u;       // (beyond every range: zeros)
      if (!TR && j == 0) inner = granule * 8;
    }
  }
  // Load j of the next unit, whose first step has place `stage` in the ring at `ring`; zeros beyond the operand.
  // By hand: with the compiler's own instruction every transposing read waits for all loads.  No register is written; vmcnt
  // counts the loads, and direct_product waits for them ahead of the barrier behind which their bytes are read.
  __device__ __forceinline__ void load(uint32_t ring, int stage, int j, int wave) const {
    typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
    const int64_t bytes = sum > 0 ? left : 0;
    const uint64_t b = reinterpret_cast<uint64_t>(base);
    const uint4v rsrc = {(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)b), (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(b >> 32)) & 0xffff,
                         (uint32_t)__builtin_amdgcn_readfirstlane(bytes < 0x7fffffff ? (uint32_t)bytes : 0x7fffffffu), 0x00027000u};
    const uint32_t own = ring + stage * kStageBytes + (wave * kLoads + j) * 1024;
    // (two instructions of a wavefront are eight rows apart, and every other one is swizzled differently)
    const int in = (j & 1) ? inner ^ 16 : inner;
    const uint32_t v = !TR && in >= sum ? 0x80000000u : at[j];
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(own), "v"(v), "s"(rsrc) : "memory", "m0");
  }
  __device__ __forceinline__ void advance() {
    base += step;
    left -= step;
    sum -= kUnit * kStep;
  }
  // Operand of one 32 x 32 x 16 instruction: 32 rows from row0, 16 of the step from k0 (0 or 16)
  static __device__ __forceinline__ bf16x8 read(const char* ring, int stage, int row0, int k0, int lane) {
    if constexpr (!TR) {
      const int r = row0 + (lane & 31);
      return *reinterpret_cast<const bf16x8*>(ring + (stage & 2) * kStageBytes + (stage & 1) * 512 + (r >> 3) * 1024 + (r & 7) * 64 +
                                              (((k0 >> 3) + (lane >> 5)) ^ row_swizzle(r)) * 16);
    } else {
      const int k = k0 + (lane >> 5) * 8 + ((lane & 15) >> 2), c = row0 + (lane & 16) + (lane & 3) * 4;
      using L = __attribute__((address_space(3))) short4v;
      union { short4v h[2]; bf16x8 x; } r;
      // (rows k and k + 4 are swizzled alike)
      const char* p = ring + stage * kStageBytes + k * (ROWS * 2) + ((c >> 3) ^ (2 * sum_swizzle(k) % kLanes)) * 16 + (c & 7) * 2;
      r.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((L*)p);
      r.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((L*)(p + 4 * ROWS * 2));
      return r.x;
    }
  }
};

// acc[tm][tn] = (A B)^T tile by tile, over all steps: a lane holds four neighbouring columns of one row at a time.  total_b: B's length of the
// summed index where A's, padded with zeros, is longer.
//
// Two instructions' worth of operands: one is multiplied while the other is read.  What a wavefront issues besides its products
// stands singly between them: a row of LDS reads or loads holds up the wavefront, and with it the matrix core (8192^3 in
// wavefronts of 128 x 128: 1950 cycles a step that way, 1450 this way; its products take 1024).
template <bool TRA, bool TRB, int WM, int WN, int TM, int TN>
__device__ __forceinline__ void direct_product(const __bf16* A, int64_t lda, int rows, const __bf16* B, int64_t ldb, int cols, int64_t total,
                                               char* smem, floatx16 (&acc)[TM][TN], int64_t total_b = 0) {
  constexpr int BM = WM * TM * 32, BN = WN * TN * 32;
  using OA = DirectOperand<TRA, BM, WM * WN>;
  using OB = DirectOperand<TRB, BN, WM * WN>;
  // loads a wavefront issues for each step, and for each two
  constexpr int kSingle = (TRA ? OA::kLoads : 0) + (TRB ? OB::kLoads : 0), kDouble = (TRA ? 0 : OA::kLoads) + (TRB ? 0 : OB::kLoads);
  const int tid = this_thread(), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int ra = (wave / WN) * TM * 32, rb = (wave % WN) * TN * 32;
#pragma unroll
  for (int tm = 0; tm < TM; ++tm)
#pragma unroll
    for (int tn = 0; tn < TN; ++tn)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[tm][tn][v] = 0.f;
  if (total <= 0) return;
  OA oa;
  OB ob;
  oa.init(A, lda, rows, (int)total, lane, wave);
  ob.init(B, ldb, cols, (int)(total_b ? total_b : total), lane, wave);
  const uint32_t lds_a = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)smem), lds_b = lds_a + OA::kBytes;
  const char* ring_a = smem;
  const char* ring_b = smem + OA::kBytes;
  // loads of a single step, of two: the j-th into the place of `stage`
  auto load_single = [&](int stage, int j) {
    if (TRA && j < OA::kLoads) oa.load(lds_a, stage, j, wave);
    else ob.load(lds_b, stage, TRA ? j - OA::kLoads : j, wave);
  };
  auto load_double = [&](int stage, int j) {
    if (!TRA && j < OA::kLoads) oa.load(lds_a, stage, j, wave);
    else ob.load(lds_b, stage, !TRA ? j - OA::kLoads : j, wave);
  };
  auto advance_single = [&] { if (TRA) oa.advance(); if (TRB) ob.advance(); };
  auto advance_double = [&] { if (!TRA) oa.advance(); if (!TRB) ob.advance(); };
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) {      // (the last single step's loads stand in the first step)
#pragma unroll
    for (int j = 0; j < kSingle; ++j) load_single(s, j);
    advance_single();
    if (s == 2) break;
#pragma unroll
    for (int j = 0; j < kDouble; ++j) load_double(2 * s, j);
    advance_double();
  }
  bf16x8 xa[2][TM], xb[2][TN];
  auto read = [&](int slot, int stage, int k0, int i) {       // in the order of use
    if (i == 0) xa[slot][0] = OA::read(ring_a, stage, ra, k0, lane);
    else if (i <= TN) xb[slot][i - 1] = OB::read(ring_b, stage, rb + (i - 1) * 32, k0, lane);
    else xa[slot][i - TN] = OA::read(ring_a, stage, ra + (i - TN) * 32, k0, lane);
  };
  constexpr int kProducts = TM * TN, kReads = TM + TN;
  auto multiply = [&](int slot, int i) {
    acc[i / TN][i % TN] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(xb[slot][i % TN], xa[slot][i / TN], acc[i / TN][i % TN], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  };
  asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(2 * kSingle + kDouble) : "memory");
#pragma unroll
  for (int i = 0; i < kReads; ++i) read(0, 0, 0, i);
  const int steps = (int)((total + kStep - 1) / kStep);
  int pair = 0;                                // place of the two steps of a turn: 0 or 2
  for (int t = 0; t < steps; t += 2) {
#pragma unroll
    for (int odd = 0; odd < 2; ++odd) {
      const int stage = pair + odd;
      // The step's first sixteen; beside them the reads for its second, and single loads three steps ahead
      constexpr int kFirst = kReads + kSingle;
#pragma unroll
      for (int i = 0; i < kProducts; ++i) {
        multiply(0, i);
#pragma unroll
        for (int j = i * kFirst / kProducts; j < (i + 1) * kFirst / kProducts; ++j) {
          if (j < kReads) read(1, stage, 16, j);
          else load_single((stage + 3) & 3, j - kReads);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      advance_single();
      // The second; beside them the reads for the next step, and behind two steps the loads of the next two but two.  Behind the barrier everybody
      // has read all of this step, so that its place is free, and everybody's loads of the next have arrived.
      constexpr int kSecond = kReads + kDouble;
#pragma unroll
      for (int i = 0; i < kProducts; ++i) {
        multiply(1, i);
        if (i == 0) {
          if (odd) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(2 * kSingle) : "memory");
          else if (kSingle) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(2 * kSingle + kDouble) : "memory");
        }
        const int n = odd ? kSecond : kReads;
#pragma unroll
        for (int j = i * n / kProducts; j < (i + 1) * n / kProducts; ++j) {
          if (j < kReads) read(0, odd ? pair ^ 2 : stage + 1, 0, j);
          else load_double(pair, j - kReads);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    advance_double();
    pair ^= 2;
  }
  // nothing may still be on its way into LDS when it is used for something else
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Results -> memory: every wavefront turns its tile through LDS (a place of its own, rows of 16 bytes more than they
// have, against the banks), so that a lane stores eight neighbouring columns and a wavefront whole lines.
template <int WM, int WN, int TM, int TN>
__device__ __forceinline__ void direct_store(const GroupedArgs& a, const GroupTile& t, int64_t c0, int rows, int cols, char* smem,
                                             const floatx16 (&acc)[TM][TN]) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int ra = (wave / WN) * TM * 32, rb = (wave % WN) * TN * 32;
  constexpr int kPitch = TN * 32 * 2 + 16, kPerRow = TN * 4;
  char* own = smem + wave * (TM * 32 * kPitch);
  const bool relu = a.act == SAGNN_ACT_RELU;
#pragma unroll
  for (int tm = 0; tm < TM; ++tm)
#pragma unroll
    for (int tn = 0; tn < TN; ++tn)
#pragma unroll
      for (int v = 0; v < 16; v += 4) {
        bf16x4 y;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float x = acc[tm][tn][v + i];
          if (relu && x < 0.f) x = 0.f;
          y[i] = (__bf16)x;
        }
        *reinterpret_cast<bf16x4*>(own + (tm * 32 + (lane & 31)) * kPitch + (tn * 32 + 2 * v + 4 * (lane >> 5)) * 2) = y;
      }
  __bf16* Y = reinterpret_cast<__bf16*>(a.Y) + t.r0 * a.ldy + c0;
  const __bf16* mask = a.mask ? reinterpret_cast<const __bf16*>(a.mask) + t.r0 * a.ldmask + c0 : nullptr;
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");        // (its own writes only)
  constexpr int kEach = TM * 32 * kPerRow / 64, kBatch = kEach < 16 ? kEach : 16;
#pragma unroll
  for (int u0 = 0; u0 < kEach; u0 += kBatch) {
    bf16x8 z[kBatch];
    if (mask) {                                              // (sixteen loads in flight; outside the tile the last row's or column's)
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int u = (u0 + b) * 64 + lane, r = ra + u / kPerRow, c = rb + u % kPerRow * 8;
        z[b] = *reinterpret_cast<const bf16x8*>(mask + (int64_t)(r < rows ? r : rows - 1) * a.ldmask + (c < cols ? c : cols - 8));
      }
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int u = (u0 + b) * 64 + lane, r = u / kPerRow, c = u % kPerRow * 8;
      bf16x8 y = *reinterpret_cast<const bf16x8*>(own + r * kPitch + c * 2);
      if (mask)
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = (float)z[b][i] > 0.f ? y[i] : (__bf16)0.f;
      if (ra + r < rows && rb + c < cols) *reinterpret_cast<bf16x8*>(Y + (int64_t)(ra + r) * a.ldy + rb + c) = y;
    }
  }
}

// LDS for a tile, with or without results that turn in it
constexpr int direct_lds(int bm, int bn, int wn) {
  const int stages = kStages * (bm + bn) * kStep * 2, out = bm * wn * (bn / wn * 2 + 16);
  return stages > out ? stages : out;
}

// A tile of 2 x WN wavefronts' rows and columns; the last tile of a group, where it has half of the rows or fewer, is
// shared by the wavefronts along the columns instead.
template <bool WT, int WN, int TM, int TN>
__device__ __forceinline__ void direct_rows_tile(const GroupedArgs& a, int32_t block, char* smem) {
  constexpr int BM = 2 * TM * 32, BN = WN * TN * 32;
  GroupTile t;
  int32_t col;
  if (!grouped_find<BM>(a, block, t, col)) return;
  const int64_t c0 = (int64_t)col * BN;
  const int rows = (int)(t.end - t.r0 < BM ? t.end - t.r0 : BM), cols = (int)(a.nout - c0 < BN ? a.nout - c0 : BN);
  const __bf16* W = reinterpret_cast<const __bf16*>(a.W) + (t.g < a.groups ? t.g * a.stride_w : 0) + c0 * (WT ? a.ldw : 1);
  const __bf16* X = reinterpret_cast<const __bf16*>(a.X) + t.r0 * a.ldx;
  const int64_t sum = t.g < a.groups ? a.kdim : 0;
  if (rows > BM / 2) {
    floatx16 acc[TM][TN];
    direct_product<false, !WT, 2, WN, TM, TN>(X, a.ldx, rows, W, a.ldw, cols, sum, smem, acc);
    direct_store<2, WN, TM, TN>(a, t, c0, rows, cols, smem, acc);
  } else {
    floatx16 acc[TM][TN / 2];
    direct_product<false, !WT, 1, 2 * WN, TM, TN / 2>(X, a.ldx, rows, W, a.ldw, cols, sum, smem, acc);
    direct_store<1, 2 * WN, TM, TN / 2>(a, t, c0, rows, cols, smem, acc);
  }
}

// A tile of the weight gradient: one group's rows of one chunk
template <int WN, int TM, int TN>
__device__ __forceinline__ void direct_tn_tile(const GroupedArgs& a, int32_t block, char* smem) {
  constexpr int BM = 2 * TM * 32, BN = WN * TN * 32;
  GroupPart p;
  int32_t tile;
  if (!grouped_part(a, block, p, tile)) return;
  const int64_t k0 = (int64_t)(tile / a.col_tiles) * BM, c0 = (int64_t)(tile % a.col_tiles) * BN;
  const int rows = (int)(a.kdim - k0 < BM ? a.kdim - k0 : BM), cols = (int)(a.nout - c0 < BN ? a.nout - c0 : BN);
  floatx16 acc[TM][TN];
  float* out = (p.cut ? a.partial + grouped_partial_slot(p) * a.kdim * a.nout : a.dW + (int64_t)p.g * a.kdim * a.nout) + k0 * a.nout + c0;
  const GroupedSides<__bf16> in(a);
  const __bf16 *X = in.X + p.r0 * in.ldx + k0, *G = in.G + p.r0 * in.ldg + c0;
  const int32_t sum = (int32_t)(p.r1 - p.r0), each = run_length(sum, a.run);
#pragma unroll 1
  for (int32_t from = 0;; from += each) {
    const bool last = sum - from <= each;
    direct_product<true, true, 2, WN, TM, TN>(X + from * in.ldx, in.ldx, rows, G + from * in.ldg, in.ldg, cols, last ? sum - from : each, smem, acc);
    const int tid = this_thread(), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ra = (wave / WN) * TM * 32 + (lane & 31), rb = (wave % WN) * TN * 32 + 4 * (lane >> 5);
#pragma unroll
    for (int tm = 0; tm < TM; ++tm) {
      // (nout is a multiple of 8: four columns are there or not)
      float* row = out + (int64_t)(ra + tm * 32) * a.nout + rb;
      if (from > 0 && ra + tm * 32 < rows && rb < cols) {      // (on top of the runs before, which are where they will be: no registers are left for them)
        float4 before[TN][4];
#pragma unroll
        for (int i = 0; i < TN * 4; ++i) before[i / 4][i % 4] = *reinterpret_cast<const float4*>(row + (rb + i * 8 < cols ? i * 8 : 0));
#pragma unroll
        for (int i = 0; i < TN * 16; ++i) acc[tm][i / 16][i % 16] += reinterpret_cast<const float*>(&before[i / 16][i % 16 / 4])[i % 4];
      }
#pragma unroll
      for (int i = 0; i < TN * 4; ++i)
        if (ra + tm * 32 < rows && rb + i * 8 < cols)
          *reinterpret_cast<float4*>(row + i * 8) =
              make_float4(acc[tm][i / 4][i % 4 * 4], acc[tm][i / 4][i % 4 * 4 + 1], acc[tm][i / 4][i % 4 * 4 + 2], acc[tm][i / 4][i % 4 * 4 + 3]);
    }
    if (last) break;
  }
}

template <bool WT, int WN, int TM, int TN>
__global__ __launch_bounds__(2 * WN * 64) void grouped_direct_kernel(const GroupedArgs a) {
  __shared__ __attribute__((aligned(1024))) char smem[direct_lds(2 * TM * 32, WN * TN * 32, WN)];
  direct_rows_tile<WT, WN, TM, TN>(a, a.first + (int32_t)blockIdx.x, smem);
}
template <int WN, int TM, int TN>
__global__ __launch_bounds__(2 * WN * 64) void grouped_direct_tn_kernel(const GroupedArgs a) {
  __shared__ __attribute__((aligned(1024))) char smem[direct_lds(2 * TM * 32, WN * TN * 32, WN)];
  direct_tn_tile<WN, TM, TN>(a, a.first + (int32_t)blockIdx.x, smem);
}
// Both gradients of a product in one launch, whose last tiles leave CUs idle once instead of twice: first `tn_blocks` for the weights,
// whose tiles are the long ones, then those for the rows (16384 x 2048 x 1024 in 16 uneven groups, calls: dX alone 98 us, dW 121, both 210 to 215).
template <int WN, int TM, int TN>
__global__ __launch_bounds__(2 * WN * 64) void grouped_direct_bwd_kernel(const GroupedArgs rows, const GroupedArgs tn, int32_t tn_blocks) {
  __shared__ __attribute__((aligned(1024))) char smem[direct_lds(2 * TM * 32, WN * TN * 32, WN)];
  const int32_t block = (int32_t)blockIdx.x;
  if (block < tn_blocks) direct_tn_tile<WN, TM, TN>(tn, block, smem);
  else direct_rows_tile<true, WN, TM, TN>(rows, block - tn_blocks, smem);
}

}  // namespace sagnn
