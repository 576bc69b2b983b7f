// Softmax cross entropy of a linear layer, logits not kept: products of rows with epilogues of their own.  One source file per
// operand mode instantiates them.
//
//   stats   tiles of z = H W + b leave a maximum, a sum of exponentials above it and the label's z for each row and tile of columns
//   grads   tiles of z become P = g (exp(z - lse) - [class == label]), stored in the operands' type, and column sums of it
//   two     the same in two bfloat16 terms, the value and what its rounding leaves, in neighbouring rows
//   rows    dH (+)= P W^T
#pragma once
#include "grouped.h"

namespace sagnn {

enum XentMode { kXentStats, kXentGrads, kXentTwo, kXentRows };

struct XentArgs {
  const void* X; int64_t ldx;                // rows x sum
  const void* W; int64_t ldw;                // sum x cols, or cols x sum
  int64_t m;                                 // rows at most
  const int32_t* count;                      // how many there are, on the device; NULL: m
  const void* all; int64_t ldall;            // may be NULL: what X is where *count is m
  int32_t cols, sum, run, mode;
  int32_t padded;                            // X's columns with zeros behind `sum`
  bool wide;                                 // results in rows that begin on 16 bytes, whole eights of them
  int32_t col_tiles; int64_t first;          // of the launch
  // stats, grads
  const float* bias; const int32_t* labels;  // bias of the first column on, or NULL
  int32_t class0, classes;                   // class of the first column, all classes
  float2* stats; float* z_label;             // col_tiles x m; m.  Or, with one tile of columns, NULL and
  float* loss; float* lse;                   // the results
  // grads; the rows are `map`'s
  const int32_t* map; const float* row_lse; float grad_all;
  const float* grad;                         // weights of the rows, or NULL; of the results of `rows` too
  bool outside;                              // they are no part of P
  float scale;                               // what is not in P (of bfloat16 products: the factor of all rows), of dbias and the results
  void* P; int64_t ldp; int32_t stored;      // columns that are stored, zeros behind `cols`
  float* bias_parts;                         // row tiles x cols, or NULL
  // rows: `splits` shares of the summed index, `share` of it each, with sums of their own, splits x m x cols, added to from piece to piece of the
  // classes; or, of one piece and one share, the result, rows by `map`, times `scale` and `grad`
  int32_t splits, share;
  float* sums; bool add;
  void* out; int64_t ldo;
};

// LDS of the epilogues: maxima, sums and the label's z of every row; sums of every column
constexpr int xent_lds(int wm, int wn, int tm, int tn) {
  const int rows = wm * tm * 32 * (wn * 8 + 4), cols = wn * tn * 32 * wm * 8;
  return rows > cols ? rows : cols;
}

// Bfloat16 results of a tile -> memory: every wavefront turns its own through LDS (rows of 16 bytes more than they have, against the
// banks), so that a lane stores eight neighbouring columns
// (four at a time, as the products leave them, 2 M x 128 results of 47 classes took 324 us).
template <typename C>
struct Turn {
  static constexpr int kPitch = C::TN * 32 * 2 + 16, kPerRow = C::TN * 4;
  static __device__ __forceinline__ char* own(char* smem) { return smem + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * (C::TM * 32 * kPitch); }
  static __device__ __forceinline__ void put(char* smem, int tm, int tn, int v, const float (&y)[4]) {
    const int lane = threadIdx.x & 63;
    bf16x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (__bf16)y[i];
    *reinterpret_cast<bf16x4*>(own(smem) + (tm * 32 + (lane & 31)) * kPitch + (tn * 32 + 2 * v + 4 * (lane >> 5)) * 2) = w;
  }
  // the value of a lane's row in its column `near`
  static __device__ __forceinline__ void put_one(char* smem, int tm, int near, float p) {
    const int lane = threadIdx.x & 63;
    *reinterpret_cast<__bf16*>(own(smem) + (tm * 32 + (lane & 31)) * kPitch + (near + 4 * (lane >> 5)) * 2) = (__bf16)p;
  }
  // at(row): offset of a row; `cols` whole eights
  template <typename F>
  static __device__ __forceinline__ void store(char* smem, __bf16* out, int rows, int cols, F at) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int ra = (wave / C::WN) * C::TM * 32, rb = (wave % C::WN) * C::TN * 32;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // (its own writes only)
#pragma unroll 4
    for (int u = lane; u < C::TM * 32 * kPerRow; u += 64) {
      const int r = u / kPerRow, c = u % kPerRow * 8;
      if (ra + r < rows && rb + c < cols)
        *reinterpret_cast<bf16x8*>(out + at(ra + r) + rb + c) = *reinterpret_cast<const bf16x8*>(own(smem) + r * kPitch + c * 2);
    }
  }
};

// What the rounding of a value leaves (nothing of an infinity or NaN)
__device__ __forceinline__ float rest_of(float x) {
  const float high = (float)(__bf16)x;
  return __builtin_fabsf(high) < INFINITY ? x - high : 0.f;
}

// The products of grouped.h, grouped_direct.h and grouped_staged.h by one name
template <typename S_, int PREC, bool TRB, int WM_, int WN_, int TM_, int TN_, int BK, bool LONG>
struct SmallProduct {
  using S = S_;
  static constexpr int WM = WM_, WN = WN_, TM = TM_, TN = TN_, kThreads = WM * WN * 64;
  static constexpr int kOperands = TileShape<PREC, false, WM * TM * 32, BK>::kBytes + TileShape<PREC, TRB, WN * TN * 32, BK>::kBytes;
  static constexpr bool kTransW = !TRB, kTurned = sizeof(S) == 2;
  static constexpr int kResults = kTurned ? WM * WN * TM * 32 * (TN * 64 + 16) : 0;
  static constexpr int kRest = kResults > xent_lds(WM, WN, TM, TN) ? kResults : xent_lds(WM, WN, TM, TN), kLds = kOperands > kRest ? kOperands : kRest;
  static __device__ __forceinline__ void run(const XentArgs& a, const S* A, int64_t lda, int rows, const S* B, int cols, int sum, int, char* smem, floatx16 (&acc)[TM][TN]) {
    tile_product<S, PREC, false, TRB, WM, WN, TM, TN, BK, LONG>(A, lda, rows, B, a.ldw, cols, sum, smem, acc, a.run);
  }
};

// e^x.  (x - y is formed first, exact where it matters: y's product taken off in one operation saves one of five, and overflows
// for the type's lowest values, which serve as masks.)
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }

// log of a sum of exponentials that is kept as (what is taken off, sum).  Nothing is taken off an infinite maximum: a row of -inf has a sum
// of 0 and one with +inf an infinite one, as the formula has it.
__device__ __forceinline__ float shift_of(float most) { return __builtin_fabsf(most) == INFINITY ? 0.f : most; }
__device__ __forceinline__ void join_stats(float& most, float& sum, float most2, float sum2) {
  const float up = fmaxf(most, most2), s = shift_of(up);
  const float a = sum == 0.f ? 0.f : sum * exp_of(shift_of(most) - s), b = sum2 == 0.f ? 0.f : sum2 * exp_of(shift_of(most2) - s);
  most = up;
  sum = a + b;
}
__device__ __forceinline__ float lse_of(float most, float sum) { return shift_of(most) + logf(sum); }

// Column, in the tile, of a lane's value v of its tile tn
template <typename C>
__device__ __forceinline__ int column_of(int tn, int v) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  return ((wave % C::WN) * C::TN + tn) * 32 + 8 * (v / 4) + 4 * (lane >> 5) + v % 4;
}
// Biases of a lane's columns
template <typename C, bool WHOLE>
__device__ __forceinline__ void load_bias(const XentArgs& a, int64_t c0, int cols, float (&b)[C::TN][16]) {
#pragma unroll
  for (int tn = 0; tn < C::TN; ++tn)
#pragma unroll
    for (int v = 0; v < 16; v += 4) {
      const int c = column_of<C>(tn, v);
      float x[4] = {0.f, 0.f, 0.f, 0.f};
      if (a.bias) {
        if (WHOLE || c + 4 <= cols) __builtin_memcpy(x, reinterpret_cast<const Four<float>*>(a.bias + c0 + c), 16);
        else
#pragma unroll
          for (int i = 0; i < 3; ++i)
            if (c + i < cols) x[i] = a.bias[c0 + c + i];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) b[tn][v + i] = x[i];
    }
}

// Whether a lane has the column `near`, counted from its first (half of the columns are those of the lane 32 away)
template <typename C>
__device__ __forceinline__ bool ours(int near) { return near >= 0 && (near & 4) == 0; }
// Of a lane's values the one of its column `near`
template <typename C>
__device__ __forceinline__ float value_at(const floatx16 (&acc)[C::TN], const float (&b)[C::TN][16], int near) {
  float x = 0.f;
#pragma unroll
  for (int tn = 0; tn < C::TN; ++tn)
#pragma unroll
    for (int v = 0; v < 16; ++v) x = near == tn * 32 + 8 * (v / 4) + v % 4 ? acc[tn][v] + b[tn][v] : x;
  return x;
}

// The epilogues take a lane's sums row by row and leave them as they are.  WHOLE: a tile without ends of the matrix, which asks nothing for each value.
template <typename C, bool WHOLE>
__device__ __forceinline__ void xent_stats(const XentArgs& a, int64_t r0, int32_t col, int64_t c0, int rows, int cols, char* smem,
                                           const floatx16 (&acc)[C::TM][C::TN]) {
  constexpr int BM = C::WM * C::TM * 32;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float b[C::TN][16];
  load_bias<C, WHOLE>(a, c0, cols, b);
  float2* place = reinterpret_cast<float2*>(smem);           // [WN][BM]
  float* z_label = reinterpret_cast<float*>(place + C::WN * BM);
#pragma unroll
  for (int tm = 0; tm < C::TM; ++tm) {
    const int r = ((wave / C::WN) * C::TM + tm) * 32 + (lane & 31);
    // the label as a number of this lane's columns
    const int64_t label = (WHOLE || r < rows ? (int64_t)a.labels[r0 + r] : -1) - c0, far = label - column_of<C>(0, 0);
    const int near = far >= 0 && far < C::TN * 32 && label < cols ? (int)far : -1;
    auto z = [&](int tn, int v) { return WHOLE || column_of<C>(tn, v) < cols ? acc[tm][tn][v] + b[tn][v] : -INFINITY; };
    const bool here = ours<C>(near);
    if (__any(here)) {                              // (few wavefronts of many classes)
      const float own = value_at<C>(acc[tm], b, near);
      if (here) (a.stats ? a.z_label + r0 : z_label)[r] = own;
    }
    float most = -INFINITY;
#pragma unroll
    for (int tn = 0; tn < C::TN; ++tn)
#pragma unroll
      for (int v = 0; v < 16; ++v) most = fmaxf(most, z(tn, v));
    most = fmaxf(most, __shfl_xor(most, 32));
    const float s = shift_of(most);
    float sum = 0.f;
#pragma unroll
    for (int tn = 0; tn < C::TN; ++tn)
#pragma unroll
      for (int v = 0; v < 16; ++v) sum += exp_of(z(tn, v) - s);
    sum += __shfl_xor(sum, 32);
    if (lane < 32) place[(wave % C::WN) * BM + r] = make_float2(most, sum);
  }
  __syncthreads();
  for (int r = threadIdx.x; r < rows; r += C::kThreads) {
    float2 p = place[r];
#pragma unroll
    for (int w = 1; w < C::WN; ++w) join_stats(p.x, p.y, place[w * BM + r].x, place[w * BM + r].y);
    if (a.stats) {
      a.stats[(int64_t)col * a.m + r0 + r] = p;
      continue;
    }
    const float lse = lse_of(p.x, p.y);
    const int32_t label = a.labels[r0 + r];
    a.lse[r0 + r] = lse;
    a.loss[r0 + r] = label >= 0 && label < a.classes ? lse - z_label[r] : 0.f;
  }
}

// Sums of what a lane holds over the sixteen lanes of its row of lanes, in every one of them
__device__ __forceinline__ float sixteen_sum(float x) {
  auto moved = [](float y, auto ctrl) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, y), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  x += moved(x, std::integral_constant<int, 0xB1>{});        // lane ^ 1
  x += moved(x, std::integral_constant<int, 0x4E>{});        // lane ^ 2
  x += moved(x, std::integral_constant<int, 0x141>{});       // the other four of eight
  x += moved(x, std::integral_constant<int, 0x140>{});       // the other eight of sixteen
  return x;
}

template <typename C, bool WHOLE, bool TWO>
__device__ __forceinline__ void xent_grads(const XentArgs& a, int64_t r0, int64_t row_tile, int64_t c0, int rows, int cols, char* smem,
                                           const floatx16 (&acc)[C::TM][C::TN]) {
  using S = typename C::S;
  constexpr int BN = C::WN * C::TN * 32;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float b[C::TN][16], sums[C::TN][16];
  load_bias<C, WHOLE>(a, c0, cols, b);
#pragma unroll
  for (int tn = 0; tn < C::TN; ++tn)
#pragma unroll
    for (int v = 0; v < 16; ++v) sums[tn][v] = 0.f;
  constexpr bool kTurned = C::kTurned && !TWO;
  const int64_t ldp = TWO ? 2 * a.ldp : a.ldp;
  S* P = reinterpret_cast<S*>(a.P) + r0 * ldp + c0;
  const int stored = a.stored - c0 < BN ? (int)(a.stored - c0) : BN;
#pragma unroll
  for (int tm = 0; tm < C::TM; ++tm) {
    const int r = ((wave / C::WN) * C::TM + tm) * 32 + (lane & 31);
    const bool in = WHOLE || r < rows;
    const int64_t row = in ? a.map[r0 + r] : 0;
    const float lse = in ? a.row_lse[row] : 0.f, own = in && a.grad ? a.grad[row] : 1.f, all = in ? a.grad_all * own : 0.f;
    const float g = a.outside ? a.grad_all : all, rest = a.outside ? own : 1.f;          // the factor in P, and that of the bias's terms
    const int64_t far = (in ? (int64_t)a.labels[row] - a.class0 : -1) - c0 - column_of<C>(0, 0);
    const int near = far >= 0 && far < C::TN * 32 && far + column_of<C>(0, 0) < cols ? (int)far : -1;
#pragma unroll
    for (int tn = 0; tn < C::TN; ++tn)
#pragma unroll
      for (int v = 0; v < 16; v += 4) {
        float y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          y[i] = exp_of(acc[tm][tn][v + i] + b[tn][v + i] - lse) * g;
          if (!WHOLE) y[i] = in && column_of<C>(tn, v + i) < cols ? y[i] : 0.f;
          sums[tn][v + i] += y[i] * rest;
        }
        if constexpr (kTurned) Turn<C>::put(smem, tm, tn, v, y);
        else if (in) store_four(P + r * ldp + column_of<C>(tn, v), y, stored - column_of<C>(tn, v));
        if constexpr (TWO)
          if (in) {
            const float low[4] = {rest_of(y[0]), rest_of(y[1]), rest_of(y[2]), rest_of(y[3])};
            store_four(P + r * ldp + a.ldp + column_of<C>(tn, v), low, stored - column_of<C>(tn, v));
          }
      }
    const bool here = ours<C>(near);
    if (__any(here)) {                              // the label's own value, over what was stored
      const float p = exp_of(value_at<C>(acc[tm], b, near) - lse) * g - g;
#pragma unroll
      for (int tn = 0; tn < C::TN; ++tn)
#pragma unroll
        for (int v = 0; v < 16; ++v) sums[tn][v] -= near == tn * 32 + 8 * (v / 4) + v % 4 ? all : 0.f;
      if (here) {
        if constexpr (kTurned) Turn<C>::put_one(smem, tm, near, p);
        else P[r * ldp + column_of<C>(0, 0) + near] = (S)p;
        if constexpr (TWO) P[r * ldp + a.ldp + column_of<C>(0, 0) + near] = (S)rest_of(p);
      }
    }
  }
  if constexpr (kTurned) Turn<C>::store(smem, P, rows, stored, [&](int r) { return r * ldp; });
  if (!a.bias_parts) return;
  // sums over the rows, of what is not rounded
  __syncthreads();
  float* place = reinterpret_cast<float*>(smem);             // [WM][2][BN]
#pragma unroll
  for (int tn = 0; tn < C::TN; ++tn)
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const float x = sixteen_sum(sums[tn][v]);
      if ((lane & 15) == 0) place[((wave / C::WN) * 2 + ((lane >> 4) & 1)) * BN + column_of<C>(tn, v)] = x;
    }
  __syncthreads();
  for (int c = threadIdx.x; c < cols; c += C::kThreads) {
    float x = 0.f;
#pragma unroll
    for (int w = 0; w < 2 * C::WM; ++w) x += place[w * BN + c];
    a.bias_parts[row_tile * a.cols + c0 + c] = x * a.scale;
  }
}

template <typename C>
__device__ __forceinline__ void xent_rows(const XentArgs& a, int32_t split, int64_t r0, int64_t c0, int rows, int cols, char* smem, floatx16 (&acc)[C::TM][C::TN]) {
  using S = typename C::S;
  if (!a.sums) {
    S* out = reinterpret_cast<S*>(a.out) + c0;
#pragma unroll
    for (int tm = 0; tm < C::TM; ++tm) {
      const int r = ((threadIdx.x >> 6) / C::WN * C::TM + tm) * 32 + (threadIdx.x & 31);
      const float factor = a.grad && r < rows ? a.scale * a.grad[a.map[r0 + r]] : a.scale;
#pragma unroll
      for (int tn = 0; tn < C::TN; ++tn)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[tm][tn][v] *= factor;
    }
    if constexpr (C::kTurned)
      if (a.wide) {
#pragma unroll
        for (int i = 0; i < C::TM * C::TN * 4; ++i) {
          const int tm = i / (C::TN * 4), tn = i / 4 % C::TN, v = i % 4 * 4;
          const float y[4] = {acc[tm][tn][v], acc[tm][tn][v + 1], acc[tm][tn][v + 2], acc[tm][tn][v + 3]};
          Turn<C>::put(smem, tm, tn, v, y);
        }
        Turn<C>::store(smem, out, rows, cols, [&](int r) { return (int64_t)a.map[r0 + r] * a.ldo; });
        return;
      }
    tile_fours<C::WM, C::WN, C::TM, C::TN>(acc, [&](int r, int c, float (&y)[4]) {
      if (r < rows) store_four(out + (int64_t)a.map[r0 + r] * a.ldo + c, y, cols - c);
    });
    return;
  }
  float* sums = a.sums + (split * a.m + r0) * a.cols + c0;
  tile_fours<C::WM, C::WN, C::TM, C::TN>(acc, [&](int r, int c, float (&y)[4]) {
    float* to = sums + (int64_t)r * a.cols + c;
    if (r >= rows) return;
    if (a.add) {
      if (c + 4 <= cols) {
        float x[4];
        __builtin_memcpy(x, reinterpret_cast<const Four<float>*>(to), 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] += x[i];
      } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
          if (c + i < cols) y[i] += to[i];
      }
    }
    store_four(to, y, cols - c);
  });
}

// Tiles in bands of eight rows of them, rows fastest, so that the tiles that an XCD has at a time share both operands' rows
constexpr int kXentBand = 8;
// X as it is for this call
struct XentRows { const void* X; int64_t ld; };
__device__ __forceinline__ XentRows xent_x(const XentArgs& a) { return a.all && *a.count == a.m ? XentRows{a.all, a.ldall} : XentRows{a.X, a.ldx}; }
struct XentTile { int64_t r0, c0; int32_t row, col, split, rows, cols, from, sum, padded; };
template <int BM, int BN>
__device__ __forceinline__ bool xent_find(const XentArgs& a, XentTile& t) {
  const int64_t m = a.count ? (*a.count < 0 ? 0 : *a.count > a.m ? a.m : *a.count) : a.m;
  const int32_t row_tiles = (int32_t)((m + BM - 1) / BM), tiles = row_tiles * a.col_tiles;
  const int64_t block = a.first + blockIdx.x, total = (int64_t)tiles * a.splits;
  if (block >= total) return false;
  int32_t id = xcd_run((int32_t)block, (int32_t)total);
  t.split = id / tiles;
  id -= t.split * tiles;
  const int32_t band = id / (kXentBand * a.col_tiles), in = id - band * kXentBand * a.col_tiles;
  const int32_t high = row_tiles - band * kXentBand < kXentBand ? row_tiles - band * kXentBand : kXentBand;
  t.row = band * kXentBand + in % high;
  t.col = in / high;
  t.r0 = (int64_t)t.row * BM;
  t.c0 = (int64_t)t.col * BN;
  t.rows = (int)(m - t.r0 < BM ? m - t.r0 : BM);
  t.cols = (int)(a.cols - t.c0 < BN ? a.cols - t.c0 : BN);
  t.from = t.split * a.share;
  t.sum = a.sum - t.from < a.share ? a.sum - t.from : a.share;
  t.padded = a.sum - t.from <= a.share ? a.padded - t.from : a.share;
  return true;
}
// (a kernel for each mode: in one for all of them the longest epilogue's registers were the products', 170 k x 128 of 172 classes 298 us for 262)
template <typename C, int MODE>
__global__ __launch_bounds__(C::kThreads, 2) void xent_kernel(const XentArgs a) {
  constexpr int BM = C::WM * C::TM * 32, BN = C::WN * C::TN * 32;
  __shared__ __attribute__((aligned(1024))) char smem[C::kLds];
  XentTile t;
  if (!xent_find<BM, BN>(a, t)) return;
  using S = typename C::S;
  floatx16 acc[C::TM][C::TN];
  const XentRows x = xent_x(a);
  C::run(a, reinterpret_cast<const S*>(x.X) + t.r0 * x.ld + t.from, x.ld, t.rows,
         reinterpret_cast<const S*>(a.W) + t.c0 * (C::kTransW ? a.ldw : 1) + (int64_t)t.from * (C::kTransW ? 1 : a.ldw), t.cols, t.sum, t.padded, smem, acc);
  __syncthreads();
  const bool whole = t.rows == BM && t.cols == BN;
  if constexpr (MODE == kXentStats) {
    if (whole) xent_stats<C, true>(a, t.r0, t.col, t.c0, t.rows, t.cols, smem, acc);
    else xent_stats<C, false>(a, t.r0, t.col, t.c0, t.rows, t.cols, smem, acc);
  } else if constexpr (MODE == kXentGrads || MODE == kXentTwo) {
    if (whole) xent_grads<C, true, MODE == kXentTwo>(a, t.r0, t.row, t.c0, t.rows, t.cols, smem, acc);
    else xent_grads<C, false, MODE == kXentTwo>(a, t.r0, t.row, t.c0, t.rows, t.cols, smem, acc);
  } else xent_rows<C>(a, t.split, t.r0, t.c0, t.rows, t.cols, smem, acc);
}

// Few rows, or few tiles for the CUs: tiles of 32 x 32, whose summed index the eight wavefronts of a workgroup share, each through LDS of its own.
// Bound by a wavefront's chain of loads, which is eight times shorter; and where a few rows meet many classes, by the weights' bytes, of which more are on
// their way (2 rows of 1831 by 39483 classes, fp32: 32 x 128 took 137 us, 2.1 TB/s).  A thread ends with two neighbouring columns of a row.
constexpr int kThinWaves = 8;
template <typename S, int PREC, bool TRB, int BK, int MODE>
__global__ __launch_bounds__(kThinWaves * 64) void xent_thin_kernel(const XentArgs a) {
  using SA = TileShape<PREC, false, 32, BK>;
  using SB = TileShape<PREC, TRB, 32, BK>;
  constexpr int kRow = 36, kSums = 32 * kRow * 4, kOwn = SA::kBytes + SB::kBytes > kSums ? SA::kBytes + SB::kBytes : kSums;
  __shared__ __attribute__((aligned(16))) char smem[kThinWaves * kOwn];
  XentTile t;
  if (!xent_find<32, 32>(a, t)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const XentRows x = xent_x(a);
  const S* X = reinterpret_cast<const S*>(x.X) + t.r0 * x.ld + t.from;
  const S* W = reinterpret_cast<const S*>(a.W) + t.c0 * (TRB ? 1 : a.ldw) + (int64_t)t.from * (TRB ? a.ldw : 1);
  TileLoad<S, PREC, false, 32, BK, 64> la;
  TileLoad<S, PREC, TRB, 32, BK, 64> lb;
  char* own = smem + wave * kOwn;
  float* sums = reinterpret_cast<float*>(smem);
  const int r = tid >> 4, c = (tid & 15) * 2;
  float y[2] = {0.f, 0.f};
  // a run of each wavefront at a time
  const int each = kThinWaves * run_length((t.sum + kThinWaves - 1) / kThinWaves, a.run);
#pragma unroll 1
  for (int from = 0; from < t.sum; from += each) {
    const int end = t.sum - from <= each ? t.sum : from + each;
    auto load = [&](int k) {
      la.load(X + k, x.ld, t.rows, end - k < BK ? end - k : BK, lane);
      lb.load(W + (int64_t)k * (TRB ? a.ldw : 1), a.ldw, t.cols, end - k < BK ? end - k : BK, lane);
    };
    floatx16 acc[1][1];
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[0][0][v] = 0.f;
    int k = from + wave * BK;
    if (k < end) load(k);
    for (; k < end; k += kThinWaves * BK) {
      la.store(own, lane);
      lb.store(own + SA::kBytes, lane);
      asm volatile("" ::: "memory");                // (a wavefront's own LDS accesses are in order)
      if (k + kThinWaves * BK < end) load(k + kThinWaves * BK);
      tile_multiply<PREC, false, TRB, 1, 1, 1, 1, BK>(own, own + SA::kBytes, acc, lane);
      asm volatile("" ::: "memory");
    }
    __syncthreads();
#pragma unroll
    for (int v = 0; v < 16; v += 4)
      *reinterpret_cast<float4*>(sums + (wave * 32 + (lane & 31)) * kRow + 2 * v + 4 * (lane >> 5)) =
          make_float4(acc[0][0][v], acc[0][0][v + 1], acc[0][0][v + 2], acc[0][0][v + 3]);
    __syncthreads();
    float all[2] = {0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kThinWaves; ++w) {
      const float2 x = *reinterpret_cast<const float2*>(sums + (w * 32 + r) * kRow + c);
      all[0] += x.x; all[1] += x.y;
    }
    y[0] += all[0]; y[1] += all[1];
    __syncthreads();                              // (the sums lie where the next run's operands do)
  }
  const bool in = r < t.rows;
  if constexpr (MODE == kXentRows) {
    float* to = a.sums ? a.sums + (t.split * a.m + t.r0 + r) * a.cols + t.c0 + c : nullptr;
    const int64_t row = in && !to ? (int64_t)a.map[t.r0 + r] : 0;
    const float factor = a.grad && in && !to ? a.scale * a.grad[row] : a.scale;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (in && c + i < t.cols) {
        if (!to) reinterpret_cast<S*>(a.out)[row * a.ldo + t.c0 + c + i] = (S)(y[i] * factor);
        else to[i] = a.add ? to[i] + y[i] : y[i];
      }
    return;
  }
  const int64_t row = !in ? 0 : MODE != kXentStats ? (int64_t)a.map[t.r0 + r] : t.r0 + r;
  const int64_t label = (in ? (int64_t)a.labels[row] - a.class0 : -1) - t.c0;
#pragma unroll
  for (int i = 0; i < 2; ++i) y[i] = c + i < t.cols ? y[i] + (a.bias ? a.bias[t.c0 + c + i] : 0.f) : -INFINITY;
  if constexpr (MODE == kXentStats) {
    float most = fmaxf(y[0], y[1]);
    for (int d = 1; d < 16; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
    const float s = shift_of(most), sum = sixteen_sum(exp_of(y[0] - s) + exp_of(y[1] - s));
    const bool here = label >= 0 && label < t.cols && (label & ~1) == c;
    const float z = sixteen_sum(here ? y[label & 1] : 0.f);                   // (all other lanes' are zeros)
    if (!in) return;
    if (a.stats) {
      if (here) a.z_label[row] = y[label & 1];
      if ((tid & 15) == 0) a.stats[(int64_t)t.col * a.m + row] = make_float2(most, sum);
    } else if ((tid & 15) == 0) {
      const float lse = lse_of(most, sum);
      a.lse[row] = lse;
      a.loss[row] = label >= 0 && label < a.classes ? lse - z : 0.f;
    }
  } else {
    const float lse = in ? a.row_lse[row] : 0.f, own = in && a.grad ? a.grad[row] : 1.f, all = in ? a.grad_all * own : 0.f;
    const float g = a.outside ? a.grad_all : all, rest = a.outside ? own : 1.f;
    S* P = reinterpret_cast<S*>(a.P) + (t.r0 + r) * (MODE == kXentTwo ? 2 * a.ldp : a.ldp) + t.c0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      y[i] = in && c + i < t.cols ? exp_of(y[i] - lse) * g - (label == c + i ? g : 0.f) : 0.f;
      if (in && t.c0 + c + i < a.stored) {
        P[c + i] = (S)y[i];
        if constexpr (MODE == kXentTwo) P[a.ldp + c + i] = (S)rest_of(y[i]);
      }
    }
    if (!a.bias_parts) return;
    *reinterpret_cast<float2*>(sums + r * kRow + c) = make_float2(y[0] * rest, y[1] * rest);
    __syncthreads();
    if (tid < t.cols) {
      float x = 0.f;
#pragma unroll 8
      for (int i = 0; i < 32; ++i) x += sums[i * kRow + tid];
      a.bias_parts[(int64_t)t.row * a.cols + t.c0 + tid] = x * a.scale;
    }
  }
}

// dW of bfloat16 tensors, rounded once where it belongs: out (rows x cols) = A^T B over the listed rows.  A and B are H and P in either order, both in rows on 16
// bytes whose ends are padded with zeros; where *count is m, the other two.
struct XentWeightArgs {
  const void *A, *B, *A2, *B2;
  int64_t lda, ldb, lda2, ldb2;
  const int32_t* count; int64_t m;
  int32_t rows, cols, row_tiles, col_tiles;
  void* out; int64_t ldo; bool wide;
  float scale;                               // of the result
};
int xent_weights_bf16(const XentWeightArgs& a, hipStream_t s);

#define SAGNN_XENT_MODE(name) int xent_##name(const XentArgs& a, int tile, bool trans_w, hipStream_t s);
SAGNN_XENT_MODE(fp32)
SAGNN_XENT_MODE(fp32_bf16)
SAGNN_XENT_MODE(fp32_bf16x3)
SAGNN_XENT_MODE(bf16)
#undef SAGNN_XENT_MODE

// launch(arguments, grid), several times where there are more tiles of `rows` rows than one launch takes
template <typename F>
int xent_launches(XentArgs a, int rows, int threads, F launch) {
  const int64_t blocks = ceil_div(a.m, rows) * a.col_tiles * a.splits, most = most_blocks(threads) / 8 * 8;
  for (a.first = 0; a.first < blocks; a.first += most) {
    launch(a, dim3((uint32_t)(blocks - a.first < most ? blocks - a.first : most)));
    SAGNN_LAUNCH_CHECK();
  }
  return SAGNN_OK;
}
template <typename C>
int xent_launch(const XentArgs& args, hipStream_t s) {
  return xent_launches(args, C::WM * C::TM * 32, C::kThreads, [&](const XentArgs& a, dim3 grid) {
    if constexpr (sizeof(typename C::S) == 2)
      if (a.mode == kXentTwo) {
        xent_kernel<C, kXentTwo><<<grid, C::kThreads, 0, s>>>(a);
        return;
      }
    if (a.mode == kXentStats) xent_kernel<C, kXentStats><<<grid, C::kThreads, 0, s>>>(a);
    else if (a.mode == kXentGrads) xent_kernel<C, kXentGrads><<<grid, C::kThreads, 0, s>>>(a);
    else xent_kernel<C, kXentRows><<<grid, C::kThreads, 0, s>>>(a);
  });
}
template <typename S, int PREC, int BK, bool TRB>
int xent_thin(const XentArgs& args, hipStream_t s) {
  return xent_launches(args, 32, kThinWaves * 64, [&](const XentArgs& a, dim3 grid) {
    if constexpr (sizeof(S) == 2)
      if (a.mode == kXentTwo) {
        xent_thin_kernel<S, PREC, TRB, BK, kXentTwo><<<grid, kThinWaves * 64, 0, s>>>(a);
        return;
      }
    if (a.mode == kXentStats) xent_thin_kernel<S, PREC, TRB, BK, kXentStats><<<grid, kThinWaves * 64, 0, s>>>(a);
    else if (a.mode == kXentGrads) xent_thin_kernel<S, PREC, TRB, BK, kXentGrads><<<grid, kThinWaves * 64, 0, s>>>(a);
    else xent_thin_kernel<S, PREC, TRB, BK, kXentRows><<<grid, kThinWaves * 64, 0, s>>>(a);
  });
}
template <typename S, int PREC, int BK, bool TRB, bool LONG>
int xent_small_as(const XentArgs& a, int tile, hipStream_t s) {
  if (tile == kTile128) return xent_launch<SmallProduct<S, PREC, TRB, 2, 2, 2, 2, BK, LONG>>(a, s);
  if (tile == kTile128x64) return xent_launch<SmallProduct<S, PREC, TRB, 2, 2, 2, 1, BK, LONG>>(a, s);
  return xent_launch<SmallProduct<S, PREC, TRB, 1, 4, 1, 1, BK, LONG>>(a, s);
}
template <typename S, int PREC, int BK>
int xent_small(const XentArgs& a, int tile, bool trans_w, hipStream_t s) {
  const bool several = a.share > a.run;
  constexpr int kThinStep = BK == 32 && PREC != SAGNN_GEMM_FP32 ? 16 : BK;
  if (tile == kThin) return trans_w ? xent_thin<S, PREC, kThinStep, false>(a, s) : xent_thin<S, PREC, kThinStep, true>(a, s);
  if (trans_w) return several ? xent_small_as<S, PREC, BK, false, true>(a, tile, s) : xent_small_as<S, PREC, BK, false, false>(a, tile, s);
  return several ? xent_small_as<S, PREC, BK, true, true>(a, tile, s) : xent_small_as<S, PREC, BK, true, false>(a, tile, s);
}

}  // namespace sagnn
