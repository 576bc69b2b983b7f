// The grouped products of fp32 tensors on the bfloat16 matrix cores in large tiles: operands pass through registers, where they are
// rounded or split, into two places in LDS.
//
// Bound: the matrix cores (six products for each of the split mode) and beside them the conversion, some seven instructions for each
// staged value, which a wavefront does between its products: those leave it seven issue slots each.  256 x 128 converts a
// quarter less than 128 x 128.  8192 x 4096 x 4096, three terms: 1340 to 1380 us, some 202 TFLOP/s, six times that on the matrix cores, the
// rate of the library's bfloat16 product.  Rounded 530 to 590 us, dX 700, less than half of that rate: one conversion for two
// values, but the same loads through registers, LDS writes and barriers for a sixth of the products.  (grouped.h's tiles of 128 x 128: 1550
// and 600.  With fp32 instructions, 133 TFLOP/s in either, there is nothing to gain.)
#pragma once
#include "grouped.h"

namespace sagnn {

constexpr int kStagedStep = 32;      // of the summed index

// An operand's tile in LDS: ROWS rows of 32 (TR: 32 rows of ROWS, the order of memory), without gaps.  Sixteen bytes are a granule;
// where it lies in its row depends on the row, so that what a read takes at once spreads over the 64 banks.
template <int PREC, bool TR, int ROWS, int THREADS>
struct StagedOperand {
  static constexpr int kPlanes = PREC == SAGNN_GEMM_FP32_BF16X3 ? 3 : 1;
  static constexpr int kPlane = ROWS * kStagedStep * 2, kBytes = kPlanes * kPlane;
  static constexpr int kPerRow = (TR ? ROWS : kStagedStep) / 4;             // units of four values along a row of memory
  static constexpr int kUnits = ROWS * kStagedStep / 4 / THREADS;           // a thread and step
  static constexpr int kApart = THREADS / kPerRow;                          // rows between a thread's units
  static_assert(kUnits * THREADS * 4 == ROWS * kStagedStep && kApart * kPerRow == THREADS, "a step must be whole units of every thread");
  const char* base;      // corner of the next step to be loaded
  int64_t step, left;    // bytes to the one after it, to the end of the operand's last row
  int sum, kept;         // of the summed index, from the next step on; in the step that the registers hold
  uint32_t at, apart;    // of this thread's first unit, between two
  int outer, inner;      // of the first unit
  float4 v[kUnits];

  __device__ __forceinline__ void init(const float* corner, int64_t ld, int rows, int total) {
    base = reinterpret_cast<const char*>(corner);
    step = TR ? kStagedStep * ld * 4 : kStagedStep * 4;
    left = ((int64_t)((TR ? total : rows) - 1) * ld + (TR ? rows : total)) * 4;
    sum = total;
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    outer = tid / kPerRow;
    inner = tid % kPerRow * 4;
    at = (uint32_t)(outer * ld + inner) * 4;
    apart = (uint32_t)(kApart * ld * 4);
  }
  // Unit u of the next step into registers.  Beyond the operand's last row zeros; beyond the summed index inside a row whatever
  // follows, which store() takes out; beyond the rows whatever follows, which is no part of a result.
  __device__ __forceinline__ void load(int u) {
    const int64_t bytes = sum > 0 ? left : 0;
    const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, bytes < 0x7fffffff ? (int)bytes : 0x7fffffff, 0x00027000);
    v[u] = __builtin_bit_cast(float4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, at + u * apart, 0, 0));
  }
  __device__ __forceinline__ void advance() {
    kept = sum;
    base += step;
    left -= step;
    sum -= kStagedStep;
  }
  // byte of four values (row r of memory's order, from i on) in a plane
  static __device__ __forceinline__ int place(int r, int i) {
    return TR ? r * (ROWS * 2) + (((i >> 3) ^ ((r & 3) * 2)) * 16) + (i & 4) * 2 : r * 64 + (((i >> 3) ^ ((r >> 2) & 3)) * 16) + (i & 4) * 2;
  }
  __device__ __forceinline__ void store(char* tile, int u) const {
    float x[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
    if constexpr (!TR)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = inner + e < kept ? x[e] : 0.f;
    char* to = tile + place(outer + u * kApart, inner);
    bf16x4 t[3];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      __bf16 t1 = (__bf16)x[e], t2 = t1, t3 = t1;
      if constexpr (kPlanes == 3) split3(x[e], t1, t2, t3);
      t[0][e] = t1; t[1][e] = t2; t[2][e] = t3;
    }
#pragma unroll
    for (int q = 0; q < kPlanes; ++q) *reinterpret_cast<bf16x4*>(to + q * kPlane) = t[q];
  }
  // 32 rows from row0, 16 of the step from k0: the operand of one 32 x 32 x 16 instruction
  static __device__ __forceinline__ bf16x8 read(const char* tile, int plane, int row0, int k0) {
    const int lane = threadIdx.x & 63;
    const char* p = tile + plane * kPlane;
    if constexpr (!TR) {
      return *reinterpret_cast<const bf16x8*>(p + place(row0 + (lane & 31), k0 + (lane >> 5) * 8));
    } else {
      const int k = k0 + (lane >> 5) * 8 + ((lane & 15) >> 2), c = row0 + (lane & 16) + (lane & 3) * 4;
      using L = __attribute__((address_space(3))) short4v;
      union { short4v h[2]; bf16x8 x; } r;
      p += place(k, c);                     // (rows k and k + 4 are placed alike)
      r.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((L*)p);
      r.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((L*)(p + 4 * ROWS * 2));
      return r.x;
    }
  }
};

// acc = A B over the summed index; the workgroup's WM x WN wavefronts own TM x TN tiles of 32 x 32 each.  Step t is multiplied out of
// one place in LDS while step t + 1 is converted into the other and step t + 2 loaded.  LONG: runs of `run` at most, which are added in registers of
// their own.
template <int PREC, bool TRA, bool TRB, int WM, int WN, int TM, int TN, bool LONG>
__device__ __forceinline__ void staged_product(const float* A, int64_t lda, int rows, const float* B, int64_t ldb, int cols, int64_t total,
                                               char* smem, floatx16 (&acc)[TM][TN], int32_t run) {
  constexpr int THREADS = WM * WN * 64;
  using OA = StagedOperand<PREC, TRA, WM * TM * 32, THREADS>;
  using OB = StagedOperand<PREC, TRB, WN * TN * 32, THREADS>;
  constexpr int kBuffer = OA::kBytes + OB::kBytes, kUnits = OA::kUnits + OB::kUnits, P = OA::kPlanes;
#pragma unroll
  for (int tm = 0; tm < TM; ++tm)
#pragma unroll
    for (int tn = 0; tn < TN; ++tn)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[tm][tn][v] = 0.f;
  if (total <= 0) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int ra = (wave / WN) * TM * 32, rb = (wave % WN) * TN * 32;
  OA oa;
  OB ob;
  oa.init(A, lda, rows, (int)total);
  ob.init(B, ldb, cols, (int)total);
  auto load = [&](int u) { if (u < OA::kUnits) oa.load(u); else ob.load(u - OA::kUnits); };
  auto store = [&](char* to, int u) { if (u < OA::kUnits) oa.store(to, u); else ob.store(to + OA::kBytes, u - OA::kUnits); };
#pragma unroll
  for (int u = 0; u < kUnits; ++u) load(u);
  oa.advance(); ob.advance();
#pragma unroll
  for (int u = 0; u < kUnits; ++u) store(smem, u);
#pragma unroll
  for (int u = 0; u < kUnits; ++u) load(u);
  oa.advance(); ob.advance();
  __syncthreads();
  const int steps = (int)((total + kStagedStep - 1) / kStagedStep);
  int at = 0;
  // two turns of sixteen sums
  bf16x8 x[2][P][TM], y[2][P][TN];
  constexpr int kReads = P * (TM + TN);
  auto read = [&](int slot, const char* tile, int k0, int i) {
    const int q = i / (TM + TN), j = i % (TM + TN);
    if (j < TM) x[slot][q][j] = OA::read(tile, q, ra + j * 32, k0);
    else y[slot][q][j - TM] = OB::read(tile + OA::kBytes, q, rb + (j - TM) * 32, k0);
  };
#pragma unroll
  for (int i = 0; i < kReads; ++i) read(0, smem, 0, i);
  [[maybe_unused]] floatx16 all[TM][TN];
  [[maybe_unused]] int left = 0;                  // steps of the run
  if constexpr (LONG) {
    run = left = run_length((int32_t)total, run) / kStagedStep;
#pragma unroll
    for (int i = 0; i < TM * TN; ++i) all[i / TN][i % TN] = acc[i / TN][i % TN];
  }
  for (int t = 0; t < steps; ++t) {
    char *tile = smem + at * kBuffer, *other = smem + (at ^ 1) * kBuffer;
#pragma unroll
    for (int turn = 0; turn < 2; ++turn) {
      // split mode: the six products down to 2^-16 of the leading one, smallest first
      constexpr int pair[6][2] = {{2, 0}, {0, 2}, {1, 1}, {1, 0}, {0, 1}, {0, 0}};
      constexpr int kTerms = P == 3 ? 6 : 1, kProducts = kTerms * TM * TN, n = kReads + kUnits;
#pragma unroll
      for (int i = 0; i < kProducts; ++i) {
        const int s = i / (TM * TN) + 6 - kTerms, tm = i / TN % TM, tn = i % TN;
        acc[tm][tn] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y[turn][pair[s][1]][tn], x[turn][pair[s][0]][tm], acc[tm][tn], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        // behind the barrier the next step is there, and nobody reads this one any more
        if (turn == 1 && i == 0) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
        for (int j = i * n / kProducts; j < (i + 1) * n / kProducts; ++j) {
          if (j < kReads) read(turn ^ 1, turn ? other : tile, turn ? 0 : 16, j);
          else if (turn) load(j - kReads);
          else store(other, j - kReads);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    oa.advance(); ob.advance();
    at ^= 1;
    if constexpr (LONG)
      if (--left == 0) {
        left = run;
#pragma unroll
        for (int i = 0; i < TM * TN; ++i) {
          all[i / TN][i % TN] += acc[i / TN][i % TN];
#pragma unroll
          for (int v = 0; v < 16; ++v) acc[i / TN][i % TN][v] = 0.f;
        }
      }
  }
  if constexpr (LONG)
#pragma unroll
    for (int i = 0; i < TM * TN; ++i) acc[i / TN][i % TN] += all[i / TN][i % TN];
}

// Tiles of WM x WN wavefronts, 64 x 64 each
template <int PREC, bool WT, int WM, int WN, bool LONG>
__global__ __launch_bounds__(WM * WN * 64) void grouped_staged_kernel(const GroupedArgs a) {
  constexpr int BM = WM * 64, BN = WN * 64, THREADS = WM * WN * 64;
  using OA = StagedOperand<PREC, false, BM, THREADS>;
  using OB = StagedOperand<PREC, !WT, BN, THREADS>;
  __shared__ __attribute__((aligned(1024))) char smem[2 * (OA::kBytes + OB::kBytes)];
  GroupTile t;
  int32_t col;
  if (!grouped_find<BM>(a, a.first + (int32_t)blockIdx.x, t, col)) return;
  const int64_t c0 = (int64_t)col * BN;
  const int rows = (int)(t.end - t.r0 < BM ? t.end - t.r0 : BM), cols = (int)(a.nout - c0 < BN ? a.nout - c0 : BN);
  const float* W = reinterpret_cast<const float*>(a.W) + (t.g < a.groups ? t.g * a.stride_w : 0) + c0 * (WT ? a.ldw : 1);
  floatx16 acc[2][2];
  staged_product<PREC, false, !WT, WM, WN, 2, 2, LONG>(reinterpret_cast<const float*>(a.X) + t.r0 * a.ldx, a.ldx, rows, W, a.ldw, cols,
                                                       t.g < a.groups ? a.kdim : 0, smem, acc, a.run);
  tile_store<float, WM, WN, 2, 2>(a, t.r0, c0, rows, cols, acc);
}

template <int PREC, int WM, int WN, bool LONG>
__global__ __launch_bounds__(WM * WN * 64) void grouped_staged_tn_kernel(const GroupedArgs a) {
  constexpr int BM = WM * 64, BN = WN * 64, THREADS = WM * WN * 64;
  using OA = StagedOperand<PREC, true, BM, THREADS>;
  using OB = StagedOperand<PREC, true, BN, THREADS>;
  __shared__ __attribute__((aligned(1024))) char smem[2 * (OA::kBytes + OB::kBytes)];
  GroupPart p;
  int32_t tile;
  if (!grouped_part(a, a.first + (int32_t)blockIdx.x, p, tile)) return;
  const int64_t k0 = (int64_t)(tile / a.col_tiles) * BM, c0 = (int64_t)(tile % a.col_tiles) * BN;
  const int rows = (int)(a.kdim - k0 < BM ? a.kdim - k0 : BM), cols = (int)(a.nout - c0 < BN ? a.nout - c0 : BN);
  floatx16 acc[2][2];
  const GroupedSides<float> in(a);
  staged_product<PREC, true, true, WM, WN, 2, 2, LONG>(in.X + p.r0 * in.ldx + k0, in.ldx, rows, in.G + p.r0 * in.ldg + c0, in.ldg, cols, p.r1 - p.r0, smem, acc,
                                                       a.run);
  float* out = (p.cut ? a.partial + grouped_partial_slot(p) * a.kdim * a.nout : a.dW + (int64_t)p.g * a.kdim * a.nout) + k0 * a.nout + c0;
  tile_fours<WM, WN, 2, 2>(acc, [&](int r, int c, float (&y)[4]) { if (r < rows) store_four(out + (int64_t)r * a.nout + c, y, cols - c); });
}

template <int PREC, int WM, int WN>
int grouped_staged_launch(const GroupedArgs& a, bool trans_w, int64_t blocks, hipStream_t s) {
  return grouped_launches(a, blocks, WM * WN * 64, [&](const GroupedArgs& part, dim3 grid) {
    const bool several = part.kdim > part.run;
    if (trans_w && several) grouped_staged_kernel<PREC, true, WM, WN, true><<<grid, WM * WN * 64, 0, s>>>(part);
    else if (trans_w) grouped_staged_kernel<PREC, true, WM, WN, false><<<grid, WM * WN * 64, 0, s>>>(part);
    else if (several) grouped_staged_kernel<PREC, false, WM, WN, true><<<grid, WM * WN * 64, 0, s>>>(part);
    else grouped_staged_kernel<PREC, false, WM, WN, false><<<grid, WM * WN * 64, 0, s>>>(part);
  });
}
template <int PREC, int WM, int WN>
int grouped_staged_tn_launch(const GroupedArgs& a, int64_t blocks, hipStream_t s) {
  return grouped_launches(a, blocks, WM * WN * 64, [&](const GroupedArgs& part, dim3 grid) {
    if (part.chunk > part.run) grouped_staged_tn_kernel<PREC, WM, WN, true><<<grid, WM * WN * 64, 0, s>>>(part);
    else grouped_staged_tn_kernel<PREC, WM, WN, false><<<grid, WM * WN * 64, 0, s>>>(part);
  });
}

}  // namespace sagnn
