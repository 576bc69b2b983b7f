// Products of rows ordered by type with a weight matrix for each type: arguments, the search for a tile's group,
// staging of operands, and the kernels that stage through registers.  One source file per operand mode instantiates them.
#pragma once
#include <initializer_list>

#include "common.h"
#include "gemm.h"

namespace sagnn {

struct GroupedArgs {
  const void* X; int64_t ldx;                    // m x kdim
  const void* W; int64_t ldw; int64_t stride_w;  // groups of kdim x nout, or nout x kdim
  const void* G; int64_t ldg;                    // weight gradient: m x nout
  const int32_t* off; int32_t groups;
  int64_t m; int32_t kdim, nout;
  int32_t act;
  const void* mask; int64_t ldmask;
  void* Y; int64_t ldy;                          // m x nout
  float* dW; float* partial;                     // weight gradient: groups x kdim x nout, sums of cut groups
  int64_t chunk;                                 // weight gradient: rows that one workgroup sums at most
  int32_t row_tiles, col_tiles;                  // of the launch
  int32_t pairs;                                 // weight gradient: numbers of pairs of a chunk and a group
  int32_t first;                                 // workgroups of the launches before this one
  int32_t run;                                   // of the summed index that one set of sums takes (grouped_run)
  const int32_t* listed;                         // weight gradient, may be NULL: where *listed is m, X and G lie elsewhere:
  const void* X2; int64_t ldx2;
  const void* G2; int64_t ldg2;
};
// The operands of a weight gradient
template <typename S>
struct GroupedSides {
  const S *X, *G;
  int64_t ldx, ldg;
  __device__ __forceinline__ explicit GroupedSides(const GroupedArgs& a) {
    const bool other = a.listed && *a.listed == a.m;
    X = reinterpret_cast<const S*>(other ? a.X2 : a.X);
    G = reinterpret_cast<const S*>(other ? a.G2 : a.G);
    ldx = other ? a.ldx2 : a.ldx;
    ldg = other ? a.ldg2 : a.ldg;
  }
};

// Sums of equal terms: every addition of a serial run may round the same way, by up to half a unit in the last place of a sum that
// grows to its end, which makes n/3 2^-24 of the whole for n additions; and the matrix cores cut off what an addend has below the sum's last
// place.  1e-5 is 168 2^-24.  Measured, the worst of millions of pairs of values: fp32 instructions 0.34 2^-24 a term; three terms 197 2^-24 for 1024
// terms and 542 for 4096 (the small products are cut first); bfloat16 0 up to 2048, where a sum of products of 16 bits begins to need
// more than 24, 128 for 4096, 192 for 6144.  A longer sum is cut into runs, which are added in turn; a run and the runs together stay below 168.
enum { kRunFp32 = 480, kRunTerms = 768, kRunBf16 = 5120 };       // a sum up to here is one run
// Bfloat16 results that the tile without room for a second set of sums makes: one run up to here, which errs by 512 2^-24 at most, a sixtieth of the
// result's own rounding (8192^3 876 us; in runs, by a smaller tile, 1578).
constexpr int64_t kRunRounded = 16384;
// The longest run of a sum of `sum`, and the longest sum
inline int32_t grouped_run(int32_t prec, int64_t sum) {
  if (prec == SAGNN_GEMM_FP32) return sum <= kRunFp32 ? kRunFp32 : sum <= 96 * 384 ? 384 : 256;
  if (prec == SAGNN_GEMM_FP32_BF16X3) return sum <= kRunTerms ? kRunTerms : 512;
  return sum <= kRunBf16 ? kRunBf16 : 4096;
}
inline int64_t grouped_sum_most(int32_t prec) {
  return prec == SAGNN_GEMM_FP32 ? 192 * 256 : prec == SAGNN_GEMM_FP32_BF16X3 ? 160 * 512 : 96 * 4096;
}
// Runs of like length, whole steps of every kernel
__device__ __forceinline__ int32_t run_length(int32_t sum, int32_t run) {
  if (sum <= run) return run;
  const int32_t runs = (sum + run - 1) / run;
  return ((sum + runs - 1) / runs + 63) & ~63;
}
// This thread's number, anew in each turn of a loop: addresses that follow from it are worked out where they are used and take no registers beside
// the products.
__device__ __forceinline__ int this_thread() {
  int t = threadIdx.x;
  asm volatile("" : "+v"(t));
  return t;
}

// Rows of group g as the kernels see them: whatever d_off holds, they lie inside [0, m).
__device__ __forceinline__ int64_t grouped_row(const int32_t* __restrict__ off, int32_t g, int64_t m) {
  const int64_t r = off[g];
  return r < 0 ? 0 : (r > m ? m : r);
}

struct GroupTile {
  int32_t g;              // == groups: the rows behind the last group
  int64_t r0, end;        // first row of the tile, end of the group
};

// Workgroups of one launch are dealt to the XCDs in turn: neighbours among n tiles go to the same one.
__device__ __forceinline__ int32_t xcd_run(int32_t id, int32_t n) {
  const int32_t each = n / 8, more = n % 8, x = id % 8;
  return x * each + (x < more ? x : more) + id / 8;
}

// Tiles of BM rows of group g, and the group's rows (g == groups: the rows behind the last group; beyond: none)
template <int BM>
__device__ __forceinline__ int32_t grouped_tiles(const GroupedArgs& a, int32_t g, int64_t& lo, int64_t& hi) {
  lo = g <= a.groups ? grouped_row(a.off, g, a.m) : 0;
  hi = g < a.groups ? grouped_row(a.off, g + 1, a.m) : (g == a.groups ? a.m : 0);
  return hi > lo ? (int32_t)((hi - lo + BM - 1) / BM) : 0;
}
// Sums of the lanes up to each, `most` at the most: ascending offsets have no more tiles than that, and others cannot wrap it.
__device__ __forceinline__ int32_t wave_sums(int32_t x, int32_t most) {
  const int lane = threadIdx.x & 63;
  if (x > most) x = most;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int32_t y = __shfl_up(x, d);
    if (lane >= d) x = x < most - y ? x + y : most;
  }
  return x;
}

// The tile of this workgroup: the groups' rows cut into tiles of BM, groups ascending, columns fastest.  How many there are only
// d_off tells, and the launch has workgroups for the most there can be; the XCDs share those that there are (dealt by
// the launch's size, the last XCDs got the missing ones: 8192^3 in five rounds instead of four).  Every wavefront looks
// for itself: 64 groups a round, a scan over the lanes.  False: no tile.
template <int BM>
__device__ __forceinline__ bool grouped_find(const GroupedArgs& a, int32_t block, GroupTile& found, int32_t& col) {
  const int lane = threadIdx.x & 63;
  int64_t lo, hi;
  int32_t tiles = grouped_tiles<BM>(a, lane, lo, hi), upto = wave_sums(tiles, a.row_tiles);
  int32_t total = __builtin_amdgcn_readlane(upto, 63);
  for (int32_t g0 = 64; g0 <= a.groups; g0 += 64) {
    int64_t l, h;
    const int32_t more = __builtin_amdgcn_readlane(wave_sums(grouped_tiles<BM>(a, g0 + lane, l, h), a.row_tiles), 63);
    total = more < a.row_tiles - total ? total + more : a.row_tiles;
  }
  if (block >= total * a.col_tiles) return false;          // (row_tiles * col_tiles is the launch's size)
  const int32_t id = xcd_run(block, total * a.col_tiles), t = id / a.col_tiles;
  col = id % a.col_tiles;
  int32_t before = 0;
  for (int32_t g0 = 0; g0 <= a.groups; g0 += 64) {
    if (g0) {
      tiles = grouped_tiles<BM>(a, g0 + lane, lo, hi);
      upto = wave_sums(tiles, a.row_tiles);
    }
    const uint64_t past = __ballot(before + upto > t);
    if (past) {
      const int f = __builtin_ctzll(past);
      const int32_t first = before + __builtin_amdgcn_readlane(upto, f) - __builtin_amdgcn_readlane(tiles, f);
      found.g = g0 + f;
      found.r0 = __builtin_amdgcn_readlane((int32_t)lo, f) + (int64_t)(t - first) * BM;
      found.end = __builtin_amdgcn_readlane((int32_t)hi, f);
      return true;
    }
    before += __builtin_amdgcn_readlane(upto, 63);
  }
  return false;
}

// The weight gradient cuts the rows into chunks whatever the groups are; a workgroup sums one group's rows of one
// chunk.  Walking along the rows, each such pair (chunk c, group g) is met at its own c + g, so that this number
// names it; not every number does.  Rows [r0, r1) of the pair that p names; cut: the group has rows in other chunks.
constexpr int32_t kManyPairs = 32;
struct GroupPart { int32_t g; int64_t r0, r1; int32_t c; bool cut, first; };
__device__ __forceinline__ bool grouped_part(const GroupedArgs& a, int32_t id, GroupPart& part, int32_t& tile) {
  const int lane = threadIdx.x & 63;
  // Tiles of a pair read the same rows.  Many pairs: an XCD has all tiles of every eighth; few: a run of the tiles of each.
  // (The last pairs may not be there, so that the XCDs share them in any case.)
  const int32_t tiles = a.row_tiles * a.col_tiles;
  int32_t p = id / tiles;
  tile = id % tiles;
  if (a.pairs >= kManyPairs) {
    p = id / 8 / tiles * 8 + id % 8;
    tile = id / 8 % tiles;
    if (p >= a.pairs) return false;
  } else if (tiles % 8 == 0) {
    tile = xcd_run(tile, tiles);
  }
  int32_t count = 0;                              // groups that begin at numbers up to p
  for (int32_t g0 = 0; g0 < a.groups; g0 += 64) {
    const int32_t g = g0 + lane;
    const int32_t begin = g < a.groups ? (int32_t)(grouped_row(a.off, g, a.m) / a.chunk) + g : INT32_MAX;
    const uint64_t upto = __ballot(begin <= p);
    count += __popcll(upto);
    if (upto != ~0ull) break;
  }
  if (count == 0) return false;
  part.g = __builtin_amdgcn_readfirstlane(count - 1);
  const int64_t lo = grouped_row(a.off, part.g, a.m), hi = grouped_row(a.off, part.g + 1, a.m);
  part.c = p - part.g;
  const int64_t c0 = lo / a.chunk, c1 = hi > lo ? (hi - 1) / a.chunk : c0;
  if (part.c < c0 || part.c > c1) return false;
  part.first = part.c == c0;
  part.cut = c1 > c0;
  part.r0 = part.first ? lo : part.c * a.chunk;
  part.r1 = hi < (part.c + 1) * a.chunk ? hi : (part.c + 1) * a.chunk;
  return true;
}

// At most one cut group runs into a chunk and one out of it, so the sum of a cut group's part has a place of its own.
__device__ __forceinline__ int64_t grouped_partial_slot(const GroupPart& p) { return 2 * (int64_t)p.c + (p.first ? 1 : 0); }

// ------------------------------------------------------------------------------------------
// Operand tiles of ROWS rows (or columns of the right operand) by BK of the summed index.  TR: the summed index is the
// outer one in memory, so a tile lies as [BK][ROWS], otherwise as [ROWS][BK]; LDS keeps the order of memory, and the
// transposition happens on the way into the matrix cores.
// A row of LDS is longer than its tile so that the reads of a wavefront spread over the banks.
template <int PREC, bool TR, int ROWS, int BK>
struct TileShape {
  static constexpr bool F32 = PREC == SAGNN_GEMM_FP32;
  static constexpr int kPlanes = PREC == SAGNN_GEMM_FP32_BF16X3 ? 3 : 1;
  static constexpr int kOuter = TR ? BK : ROWS, kInner = TR ? ROWS : BK;
  static constexpr int kPitch = F32 ? (TR ? ROWS + 8 : BK + 4) : (TR ? ROWS + 32 : BK + 8);
  static constexpr int kPlane = kOuter * kPitch;                       // elements
  static constexpr int kBytes = kPlane * kPlanes * (F32 ? 4 : 2);
};

template <typename T>
struct __attribute__((packed)) Unaligned { T v; };

template <typename S, int PREC, bool TR, int ROWS, int BK, int THREADS>
struct TileLoad {
  using Shape = TileShape<PREC, TR, ROWS, BK>;
  static constexpr int V = 16 / sizeof(S);
  static constexpr int kPerRow = Shape::kInner / V;
  static constexpr int N = Shape::kOuter * kPerRow / THREADS;
  static_assert(N * THREADS == Shape::kOuter * kPerRow, "tile and workgroup must match");
  struct __attribute__((aligned(16))) Vec { S x[V]; };
  Vec v[N];

  // the tile at `base` (leading dimension ld), of which `rows` rows and `sum` of the summed index are there (both
  // may exceed the tile; at least one of each).  Zeros beyond `sum`; rows beyond `rows` are zeros or any row's.
  __device__ __forceinline__ void load(const S* __restrict__ base, int64_t ld, int rows, int sum, int tid) {
    const int outer_end = TR ? sum : rows, inner_end = TR ? rows : sum;
    if (inner_end >= Shape::kInner && (!TR || sum >= BK)) {
#pragma unroll
      for (int u = 0; u < N; ++u) {
        const int w = tid + u * THREADS;
        int o = w / kPerRow;
        if (!TR) o = o < outer_end ? o : outer_end - 1;
        const S* p = base + (int64_t)o * ld + (w % kPerRow) * V;
        // (any element's alignment: the memory instructions take it)
        v[u] = *reinterpret_cast<const Vec*>(&reinterpret_cast<const Unaligned<Vec>*>(p)->v);
      }
      return;
    }
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int w = tid + u * THREADS, o = w / kPerRow, i = (w % kPerRow) * V;
      const int there = o < outer_end ? inner_end - i : 0;
      const S* p = base + (int64_t)o * ld + i;
      if (there >= V) {
        v[u] = *reinterpret_cast<const Vec*>(&reinterpret_cast<const Unaligned<Vec>*>(p)->v);
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e) v[u].x[e] = e < there ? p[e] : (S)0.f;
      }
    }
  }

  __device__ __forceinline__ void store(char* smem, int tid) const {
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int w = tid + u * THREADS, at = (w / kPerRow) * Shape::kPitch + (w % kPerRow) * V;
      if constexpr (PREC == SAGNN_GEMM_FP32) {
        *reinterpret_cast<Vec*>(reinterpret_cast<float*>(smem) + at) = v[u];
      } else if constexpr (sizeof(S) == 2) {
        *reinterpret_cast<Vec*>(reinterpret_cast<__bf16*>(smem) + at) = v[u];
      } else {
        bf16x4 t[3];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          __bf16 t1 = (__bf16)v[u].x[e], t2 = t1, t3 = t1;
          if constexpr (PREC == SAGNN_GEMM_FP32_BF16X3) split3(v[u].x[e], t1, t2, t3);
          t[0][e] = t1; t[1][e] = t2; t[2][e] = t3;
        }
#pragma unroll
        for (int q = 0; q < Shape::kPlanes; ++q)
          *reinterpret_cast<bf16x4*>(reinterpret_cast<__bf16*>(smem) + q * Shape::kPlane + at) = t[q];
      }
    }
  }
};

typedef short short4v __attribute__((ext_vector_type(4)));

// 32 rows (or columns) from `row0` on, 16 of the summed index from `k0` on: the operand of one 32x32x16 instruction.
// A lane has row lane % 32 and the eight sums of its half.  TR: two transposing reads; sixteen lanes read four rows of
// 32 bytes, and each gets a column of four.
template <typename Shape, bool TR>
__device__ __forceinline__ bf16x8 tile_operand(const __bf16* tile, int row0, int k0, int lane) {
  if constexpr (!TR) {
    return *reinterpret_cast<const bf16x8*>(tile + (row0 + (lane & 31)) * Shape::kPitch + k0 + (lane >> 5) * 8);
  } else {
    const __bf16* p = tile + (k0 + (lane >> 5) * 8 + ((lane & 15) >> 2)) * Shape::kPitch + row0 + (lane & 16) + (lane & 3) * 4;
    using L = __attribute__((address_space(3))) short4v;
    union { short4v h[2]; bf16x8 x; } r;
    r.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((L*)p);
    r.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((L*)(p + 4 * Shape::kPitch));
    return r.x;
  }
}

// acc += A B over one staged step.  The workgroup's WM x WN wavefronts own TM x TN tiles of 32 x 32 each.
template <int PREC, bool TRA, bool TRB, int WM, int WN, int TM, int TN, int BK>
__device__ __forceinline__ void tile_multiply(const char* sa, const char* sb, floatx16 (&acc)[TM][TN], int tid) {
  using SA = TileShape<PREC, TRA, WM * TM * 32, BK>;
  using SB = TileShape<PREC, TRB, WN * TN * 32, BK>;
  const int lane = tid & 63, wave = tid >> 6;
  const int ra = (wave / WN) * TM * 32, rb = (wave % WN) * TN * 32;
  if constexpr (PREC == SAGNN_GEMM_FP32) {
    const float* A = reinterpret_cast<const float*>(sa);
    const float* B = reinterpret_cast<const float*>(sb);
    const int r = lane & 31, h = lane >> 5;
    // eight sums a turn: the lower half of the wavefront takes the first four, the upper one the others
#pragma unroll
    for (int k = 0; k < BK; k += 8) {
      float x[TM][4], y[TN][4];
#pragma unroll
      for (int t = 0; t < TM; ++t) {
        if constexpr (!TRA) *reinterpret_cast<float4*>(x[t]) = *reinterpret_cast<const float4*>(A + (ra + t * 32 + r) * SA::kPitch + k + 4 * h);
        else
#pragma unroll
          for (int i = 0; i < 4; ++i) x[t][i] = A[(k + 4 * h + i) * SA::kPitch + ra + t * 32 + r];
      }
#pragma unroll
      for (int t = 0; t < TN; ++t) {
        if constexpr (!TRB) *reinterpret_cast<float4*>(y[t]) = *reinterpret_cast<const float4*>(B + (rb + t * 32 + r) * SB::kPitch + k + 4 * h);
        else
#pragma unroll
          for (int i = 0; i < 4; ++i) y[t][i] = B[(k + 4 * h + i) * SB::kPitch + rb + t * 32 + r];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int tm = 0; tm < TM; ++tm)
#pragma unroll
          for (int tn = 0; tn < TN; ++tn)
            acc[tm][tn] = __builtin_amdgcn_mfma_f32_32x32x2f32(y[tn][i], x[tm][i], acc[tm][tn], 0, 0, 0);
    }
  } else {
    const __bf16* A = reinterpret_cast<const __bf16*>(sa);
    const __bf16* B = reinterpret_cast<const __bf16*>(sb);
    constexpr int P = SA::kPlanes;
#pragma unroll
    for (int k = 0; k < BK; k += 16) {
      bf16x8 x[P][TM], y[P][TN];
#pragma unroll
      for (int q = 0; q < P; ++q) {
#pragma unroll
        for (int t = 0; t < TM; ++t) x[q][t] = tile_operand<SA, TRA>(A + q * SA::kPlane, ra + t * 32, k, lane);
#pragma unroll
        for (int t = 0; t < TN; ++t) y[q][t] = tile_operand<SB, TRB>(B + q * SB::kPlane, rb + t * 32, k, lane);
      }
      // split mode: the six products down to 2^-16 of the leading one, smallest first
      constexpr int pair[6][2] = {{2, 0}, {0, 2}, {1, 1}, {1, 0}, {0, 1}, {0, 0}};
#pragma unroll
      for (int s = P == 3 ? 0 : 5; s < 6; ++s)
#pragma unroll
        for (int tm = 0; tm < TM; ++tm)
#pragma unroll
          for (int tn = 0; tn < TN; ++tn)
            acc[tm][tn] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y[pair[s][1]][tn], x[pair[s][0]][tm], acc[tm][tn], 0, 0, 0);
    }
  }
}

// acc = A B over `sum` of the summed index: a step of both operands is loaded into registers while the one before it
// is multiplied out of LDS.  LONG: runs of `run` at most, which are added in registers of their own.
template <typename S, int PREC, bool TRA, bool TRB, int WM, int WN, int TM, int TN, int BK, bool LONG>
__device__ __forceinline__ void tile_product(const S* A, int64_t lda, int rows, const S* B, int64_t ldb, int cols, int64_t sum,
                                             char* smem, floatx16 (&acc)[TM][TN], int32_t run) {
  constexpr int THREADS = WM * WN * 64;
  using SA = TileShape<PREC, TRA, WM * TM * 32, BK>;
  TileLoad<S, PREC, TRA, WM * TM * 32, BK, THREADS> la;
  TileLoad<S, PREC, TRB, WN * TN * 32, BK, THREADS> lb;
#pragma unroll
  for (int tm = 0; tm < TM; ++tm)
#pragma unroll
    for (int tn = 0; tn < TN; ++tn)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[tm][tn][v] = 0.f;
  if (sum <= 0) return;
  auto left = [&](int64_t k) { return (int)(sum - k < BK ? sum - k : BK); };
  const int tid = threadIdx.x;
  [[maybe_unused]] floatx16 all[TM][TN];
  [[maybe_unused]] int64_t until = 0;             // end of the run
  if constexpr (LONG) {
    until = run = run_length((int32_t)sum, run);
#pragma unroll
    for (int i = 0; i < TM * TN; ++i) all[i / TN][i % TN] = acc[i / TN][i % TN];
  }
  la.load(A, lda, rows, left(0), tid);
  lb.load(B, ldb, cols, left(0), tid);
  for (int64_t k = 0; k < sum; k += BK) {
    la.store(smem, tid);
    lb.store(smem + SA::kBytes, tid);
    __syncthreads();
    if (k + BK < sum) {
      la.load(A + (k + BK) * (TRA ? lda : 1), lda, rows, left(k + BK), tid);
      lb.load(B + (k + BK) * (TRB ? ldb : 1), ldb, cols, left(k + BK), tid);
    }
    tile_multiply<PREC, TRA, TRB, WM, WN, TM, TN, BK>(smem, smem + SA::kBytes, acc, tid);
    __syncthreads();
    if constexpr (LONG)                           // (as a loop around this one it cost 16 % where it costs 4: 1024 x 1024, three terms)
      if (k + BK >= until) {
        until += run;
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

// f(row, column, sums) of what a lane holds, four neighbouring columns of a row at a time (the products are taken transposed for
// that), relative to the workgroup's tile
template <int WM, int WN, int TM, int TN, typename F>
__device__ __forceinline__ void tile_fours(floatx16 (&acc)[TM][TN], F f) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int tm = 0; tm < TM; ++tm)
#pragma unroll
    for (int tn = 0; tn < TN; ++tn)
#pragma unroll
      for (int v = 0; v < 16; v += 4) {
        float y[4] = {acc[tm][tn][v], acc[tm][tn][v + 1], acc[tm][tn][v + 2], acc[tm][tn][v + 3]};
        f(((wave / WN) * TM + tm) * 32 + (lane & 31), ((wave % WN) * TN + tn) * 32 + 2 * v + 4 * (lane >> 5), y);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[tm][tn][v + i] = y[i];
      }
}
// Four values at p, of which `there` are inside (any alignment)
template <typename S>
struct __attribute__((packed)) Four { S x[4]; };
template <typename S>
__device__ __forceinline__ void store_four(S* p, const float (&y)[4], int there) {
  if (there >= 4) {
    struct __attribute__((aligned(sizeof(S) * 4))) Whole { S x[4]; } w = {(S)y[0], (S)y[1], (S)y[2], (S)y[3]};
    __builtin_memcpy(reinterpret_cast<Four<S>*>(p), &w, sizeof(w));
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (i < there) p[i] = (S)y[i];
  }
}
template <typename S>
__device__ __forceinline__ void mask_four(const S* p, float (&y)[4], int there) {
  if (there >= 4) {
    struct __attribute__((aligned(sizeof(S) * 4))) Whole { S x[4]; } w;
    __builtin_memcpy(&w, reinterpret_cast<const Four<S>*>(p), sizeof(w));
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = (float)w.x[i] > 0.f ? y[i] : 0.f;
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (i < there) y[i] = (float)p[i] > 0.f ? y[i] : 0.f;
  }
}

// A tile's mask.  A lane outside takes the last row's or columns' values, so that the loads of a row of tiles are in flight together;
// behind a branch each waits for the one before (10005 x 176 by 1648 columns, three terms: 68 us without a mask, 95 that way, 75 this way).
template <typename S, int WM, int WN, int TM, int TN>
__device__ __forceinline__ void tile_mask(const S* mask, int64_t ld, int rows, int cols, floatx16 (&acc)[TM][TN]) {
  if (cols < 4) {
    tile_fours<WM, WN, TM, TN>(acc, [&](int r, int c, float (&y)[4]) { if (r < rows) mask_four(mask + (int64_t)r * ld + c, y, cols - c); });
    return;
  }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r0 = (wave / WN) * TM * 32 + (lane & 31), c0 = (wave % WN) * TN * 32 + 4 * (lane >> 5);
#pragma unroll
  for (int tm = 0; tm < TM; ++tm) {
    struct __attribute__((aligned(sizeof(S) * 4))) Whole { S x[4]; } z[TN][4];
    const int r = r0 + tm * 32 < rows ? r0 + tm * 32 : rows - 1;
#pragma unroll
    for (int tn = 0; tn < TN; ++tn)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int c = c0 + tn * 32 + 8 * v;
        __builtin_memcpy(&z[tn][v], reinterpret_cast<const Four<S>*>(mask + (int64_t)r * ld + (c < cols - 4 ? c : cols - 4)), sizeof(Whole));
      }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int tn = 0; tn < TN; ++tn)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        S (&x)[4] = z[tn][v].x;
        if (cols & 3) {                           // (four columns across the tile's end were loaded up to three too early)
          const int early = c0 + tn * 32 + 8 * v - (cols - 4);
          if (early == 1) { x[0] = x[1]; x[1] = x[2]; x[2] = x[3]; }
          if (early == 2) { x[0] = x[2]; x[1] = x[3]; }
          if (early == 3) x[0] = x[3];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (!((float)x[i] > 0.f)) acc[tm][tn][4 * v + i] = 0.f;
      }
  }
}

// Results of a tile at row r0, column c0 -> Y, through activation and mask
template <typename S, int WM, int WN, int TM, int TN>
__device__ __forceinline__ void tile_store(const GroupedArgs& a, int64_t r0, int64_t c0, int rows, int cols, floatx16 (&acc)[TM][TN]) {
  S* Y = reinterpret_cast<S*>(a.Y) + r0 * a.ldy + c0;
  const bool relu = a.act == SAGNN_ACT_RELU;
  if (a.mask)                                   // (all loads ahead of the stores, which the compiler could not pass)
    tile_mask<S, WM, WN, TM, TN>(reinterpret_cast<const S*>(a.mask) + r0 * a.ldmask + c0, a.ldmask, rows, cols, acc);
  tile_fours<WM, WN, TM, TN>(acc, [&](int r, int c, float (&y)[4]) {
    if (relu)
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = y[i] < 0.f ? 0.f : y[i];
    if (r < rows) store_four(Y + (int64_t)r * a.ldy + c, y, cols - c);
  });
}

// LONG, here and below: a sum of several runs.  (Two workgroups on a CU are worth the registers that they have to give up for it; not the
// wide steps of operands that are rounded on the way, whose sums would be spilled.)
template <typename S, int PREC, bool WT, int WM, int WN, int TM, int TN, int BK, bool LONG>
__global__ __launch_bounds__(WM * WN * 64, LONG && !(sizeof(S) == 4 && PREC == SAGNN_GEMM_BF16) ? 2 : 1) void grouped_kernel(const GroupedArgs a) {
  constexpr int BM = WM * TM * 32, BN = WN * TN * 32;
  __shared__ __attribute__((aligned(16))) char smem[TileShape<PREC, false, BM, BK>::kBytes + TileShape<PREC, !WT, BN, BK>::kBytes];
  GroupTile t;
  int32_t col;
  if (!grouped_find<BM>(a, a.first + (int32_t)blockIdx.x, t, col)) return;
  const int64_t c0 = (int64_t)col * BN;
  const int rows = (int)(t.end - t.r0 < BM ? t.end - t.r0 : BM), cols = (int)(a.nout - c0 < BN ? a.nout - c0 : BN);
  floatx16 acc[TM][TN];
  const S* W = reinterpret_cast<const S*>(a.W) + (t.g < a.groups ? t.g * a.stride_w : 0) + c0 * (WT ? a.ldw : 1);
  tile_product<S, PREC, false, !WT, WM, WN, TM, TN, BK, LONG>(reinterpret_cast<const S*>(a.X) + t.r0 * a.ldx, a.ldx, rows, W, a.ldw, cols,
                                                              t.g < a.groups ? a.kdim : 0, smem, acc, a.run);
  tile_store<S, WM, WN, TM, TN>(a, t.r0, c0, rows, cols, acc);
}

// Few rows of a group, or few tiles for the CUs: a workgroup's wavefronts share the summed index of one tile of 32 rows instead of
// the tile, each through a part of LDS of its own, and their sums are added in LDS at the end.  Bound by the chain of
// loads of a wavefront, which is WAVES times shorter (3 rows, 2211 x 228 of 28 groups: 70 us by 32 x 128, 19 this way; 44 columns' gradient for
// 1000 rows of 46 groups, 1066 deep: 36 and 12).
template <typename S, int PREC, bool WT, int TN, int WAVES, int BK>
__global__ __launch_bounds__(WAVES * 64) void grouped_thin_kernel(const GroupedArgs a) {
  constexpr int BN = TN * 32, kRow = BN + 4;
  using SA = TileShape<PREC, false, 32, BK>;
  using SB = TileShape<PREC, !WT, BN, BK>;
  constexpr int kOwn = SA::kBytes + SB::kBytes, kSums = 32 * kRow * 4;
  __shared__ __attribute__((aligned(16))) char smem[WAVES * (kOwn > kSums ? kOwn : kSums)];
  GroupTile t;
  int32_t col;
  if (!grouped_find<32>(a, a.first + (int32_t)blockIdx.x, t, col)) return;
  const int64_t c0 = (int64_t)col * BN;
  const int rows = (int)(t.end - t.r0 < 32 ? t.end - t.r0 : 32), cols = (int)(a.nout - c0 < BN ? a.nout - c0 : BN);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const S* X = reinterpret_cast<const S*>(a.X) + t.r0 * a.ldx;
  const S* W = reinterpret_cast<const S*>(a.W) + (t.g < a.groups ? t.g * a.stride_w : 0) + c0 * (WT ? a.ldw : 1);
  TileLoad<S, PREC, false, 32, BK, 64> la;
  TileLoad<S, PREC, !WT, BN, BK, 64> lb;
  const int sum = t.g < a.groups ? a.kdim : 0;
  char* own = smem + wave * kOwn;
  float* sums = reinterpret_cast<float*>(smem);
  S* Y = reinterpret_cast<S*>(a.Y) + t.r0 * a.ldy + c0;
  const S* mask = a.mask ? reinterpret_cast<const S*>(a.mask) + t.r0 * a.ldmask + c0 : nullptr;
  // a run of each wavefront at a time (bfloat16 results: there is one only)
  const int32_t each = sizeof(S) == 4 ? WAVES * run_length((sum + WAVES - 1) / WAVES, a.run) : sum;
#pragma unroll 1
  for (int32_t from = 0;; from += each) {
    const bool last = sum - from <= each;
    const int end = last ? sum : from + each;
    const int tid = this_thread(), lane = tid & 63;
    auto load = [&](int k) {
      la.load(X + k, a.ldx, rows, end - k < BK ? end - k : BK, lane);
      lb.load(W + (int64_t)k * (WT ? 1 : a.ldw), a.ldw, cols, end - k < BK ? end - k : BK, lane);
    };
    floatx16 acc[1][TN];
#pragma unroll
    for (int tn = 0; tn < TN; ++tn)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[0][tn][v] = 0.f;
    int k = from + wave * BK;
    if (k < end) load(k);
    for (; k < end; k += WAVES * BK) {
      la.store(own, lane);
      lb.store(own + SA::kBytes, lane);
      asm volatile("" ::: "memory");                // (a wavefront's own LDS accesses are in order)
      if (k + WAVES * BK < end) load(k + WAVES * BK);
      tile_multiply<PREC, false, !WT, 1, 1, 1, TN, BK>(own, own + SA::kBytes, acc, lane);
      asm volatile("" ::: "memory");
    }
    __syncthreads();
#pragma unroll
    for (int tn = 0; tn < TN; ++tn)
#pragma unroll
      for (int v = 0; v < 16; v += 4)
        *reinterpret_cast<float4*>(sums + (wave * 32 + (lane & 31)) * kRow + tn * 32 + 2 * v + 4 * (lane >> 5)) =
            make_float4(acc[0][tn][v], acc[0][tn][v + 1], acc[0][tn][v + 2], acc[0][tn][v + 3]);
    __syncthreads();
    for (int u = tid; u < 32 * (BN / 4); u += WAVES * 64) {
      const int r = u / (BN / 4), c = u % (BN / 4) * 4;
      if (r >= rows || c >= cols) continue;
      float y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        const float4 x = *reinterpret_cast<const float4*>(sums + (w * 32 + r) * kRow + c);
        y[0] += x.x; y[1] += x.y; y[2] += x.z; y[3] += x.w;
      }
      S* to = Y + (int64_t)r * a.ldy + c;
      if constexpr (sizeof(S) == 4)
        if (from > 0)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (c + i < cols) y[i] += to[i];
      if (last && a.act == SAGNN_ACT_RELU)
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = y[i] < 0.f ? 0.f : y[i];
      if (last && mask) mask_four(mask + (int64_t)r * a.ldmask + c, y, cols - c);
      store_four(to, y, cols - c);
    }
    if (last) break;
    __syncthreads();                              // (the sums lie where the next run's operands do)
  }
}

template <typename S, int PREC, int WM, int WN, int TM, int TN, int BK, bool LONG>
__global__ __launch_bounds__(WM * WN * 64, LONG && !(sizeof(S) == 4 && PREC == SAGNN_GEMM_BF16) ? 2 : 1) void grouped_tn_kernel(const GroupedArgs a) {
  constexpr int BM = WM * TM * 32, BN = WN * TN * 32;
  __shared__ __attribute__((aligned(16))) char smem[TileShape<PREC, true, BM, BK>::kBytes + TileShape<PREC, true, BN, BK>::kBytes];
  GroupPart p;
  int32_t tile;
  if (!grouped_part(a, a.first + (int32_t)blockIdx.x, p, tile)) return;
  const int64_t k0 = (int64_t)(tile / a.col_tiles) * BM, c0 = (int64_t)(tile % a.col_tiles) * BN;
  const int rows = (int)(a.kdim - k0 < BM ? a.kdim - k0 : BM), cols = (int)(a.nout - c0 < BN ? a.nout - c0 : BN);
  floatx16 acc[TM][TN];
  float* out = (p.cut ? a.partial + grouped_partial_slot(p) * a.kdim * a.nout : a.dW + (int64_t)p.g * a.kdim * a.nout) + k0 * a.nout + c0;
  const GroupedSides<S> in(a);
  tile_product<S, PREC, true, true, WM, WN, TM, TN, BK, LONG>(in.X + p.r0 * in.ldx + k0, in.ldx, rows, in.G + p.r0 * in.ldg + c0, in.ldg, cols, p.r1 - p.r0,
                                                              smem, acc, a.run);
  tile_fours<WM, WN, TM, TN>(acc, [&](int r, int c, float (&y)[4]) { if (r < rows) store_four(out + (int64_t)r * a.nout + c, y, cols - c); });
}

constexpr int kThinCols = 32;
// Tiles that a launch can take, rows of X (of W for the weight gradient) by columns
enum GroupedTile { kTile128, kTile128x64, kTile128x32, kTile64, kTile32x128, kDirect256, kStaged256x128, kStaged128x256, kThin, kGroupedTiles };
inline int grouped_tile_rows(int tile) {
  constexpr int rows[kGroupedTiles] = {128, 128, 128, 64, 32, 256, 256, 128, 32};
  return rows[tile];
}
inline int grouped_tile_cols(int tile) {
  constexpr int cols[kGroupedTiles] = {128, 64, 32, 64, 128, 256, 128, 256, kThinCols};
  return cols[tile];
}

// What a tile costs: how well it feeds the matrix cores (rates of 8192 x 4096 x 4096, 128 x 128 = 1), and how much of the summed index its
// beginning and end are worth.  Small tiles are several to a CU, which hides both; the large ones are alone there.
struct TileCost { double rate, ends; };
TileCost tile_cost(int32_t dtype, int32_t prec, int tile);

// dW of grouped_gemm_bwd for arguments that are filled in but for the launch's; ws: as much as it says
int grouped_weights(const GroupedArgs& a, int32_t dtype, int32_t prec, hipStream_t s);
// Bytes of its `partial`, of one group of m rows, for any types and modes
size_t grouped_weights_bytes(int64_t m, int32_t kdim, int32_t nout);

// a product of `blocks` workgroups; per operand mode (and storage type)
#define SAGNN_GROUPED_MODE(name)                                                                                       \
  int grouped_##name(const GroupedArgs& a, int tile, bool trans_w, int64_t blocks, hipStream_t s);                      \
  int grouped_tn_##name(const GroupedArgs& a, int tile, int64_t blocks, hipStream_t s);
SAGNN_GROUPED_MODE(fp32)
SAGNN_GROUPED_MODE(fp32_bf16)
SAGNN_GROUPED_MODE(fp32_bf16x3)
SAGNN_GROUPED_MODE(bf16)
#undef SAGNN_GROUPED_MODE
int grouped_bwd_bf16(const GroupedArgs& rows, int64_t rows_blocks, const GroupedArgs& tn, int64_t tn_blocks, hipStream_t s);

// `blocks` workgroups: launch(arguments, grid), several times where they are more than one launch takes
template <typename F>
int grouped_launches(GroupedArgs a, int64_t blocks, int threads, F launch) {
  const int64_t most = most_blocks(threads) / 8 * 8;        // (the XCDs are dealt to in turn)
  for (int64_t b = 0; b < blocks; b += most) {
    a.first = (int32_t)b;
    launch(a, dim3((uint32_t)(blocks - b < most ? blocks - b : most)));
    SAGNN_LAUNCH_CHECK();
  }
  return SAGNN_OK;
}

template <typename S, int PREC, int BK, bool WT, bool LONG>
void grouped_launch_as(const GroupedArgs& a, int tile, dim3 grid, hipStream_t s) {
  const dim3 block(256);
  if (tile == kTile128) grouped_kernel<S, PREC, WT, 2, 2, 2, 2, BK, LONG><<<grid, block, 0, s>>>(a);
  else if (tile == kTile128x64) grouped_kernel<S, PREC, WT, 2, 2, 2, 1, BK, LONG><<<grid, block, 0, s>>>(a);
  else if (tile == kTile128x32) grouped_kernel<S, PREC, WT, 4, 1, 1, 1, BK, LONG><<<grid, block, 0, s>>>(a);
  else if (tile == kTile64) grouped_kernel<S, PREC, WT, 2, 2, 1, 1, BK, LONG><<<grid, block, 0, s>>>(a);
  else grouped_kernel<S, PREC, WT, 1, 4, 1, 1, BK, LONG><<<grid, block, 0, s>>>(a);
}
template <typename S, int PREC, int BK, bool WT>
int grouped_launch(const GroupedArgs& args, int tile, int64_t blocks, hipStream_t s) {
  return grouped_launches(args, blocks, tile == kThin ? 512 : 256, [&](const GroupedArgs& a, dim3 grid) {
    if (tile == kThin) grouped_thin_kernel<S, PREC, WT, kThinCols / 32, 8, BK == 32 && PREC != SAGNN_GEMM_FP32 ? 16 : BK><<<grid, 512, 0, s>>>(a);
    else if (a.kdim > a.run) grouped_launch_as<S, PREC, BK, WT, true>(a, tile, grid, s);
    else grouped_launch_as<S, PREC, BK, WT, false>(a, tile, grid, s);
  });
}
template <typename S, int PREC, int BK, bool LONG>
void grouped_tn_launch_as(const GroupedArgs& a, int tile, dim3 grid, hipStream_t s) {
  const dim3 block(256);
  if (tile == kTile128) grouped_tn_kernel<S, PREC, 2, 2, 2, 2, BK, LONG><<<grid, block, 0, s>>>(a);
  else if (tile == kTile128x64) grouped_tn_kernel<S, PREC, 2, 2, 2, 1, BK, LONG><<<grid, block, 0, s>>>(a);
  else if (tile == kTile128x32) grouped_tn_kernel<S, PREC, 4, 1, 1, 1, BK, LONG><<<grid, block, 0, s>>>(a);
  else if (tile == kTile64) grouped_tn_kernel<S, PREC, 2, 2, 1, 1, BK, LONG><<<grid, block, 0, s>>>(a);
  else grouped_tn_kernel<S, PREC, 1, 4, 1, 1, BK, LONG><<<grid, block, 0, s>>>(a);
}
template <typename S, int PREC, int BK>
int grouped_tn_launch(const GroupedArgs& args, int tile, int64_t blocks, hipStream_t s) {
  return grouped_launches(args, blocks, 256, [&](const GroupedArgs& a, dim3 grid) {
    if (a.chunk > a.run) grouped_tn_launch_as<S, PREC, BK, true>(a, tile, grid, s);
    else grouped_tn_launch_as<S, PREC, BK, false>(a, tile, grid, s);
  });
}

}  // namespace sagnn
