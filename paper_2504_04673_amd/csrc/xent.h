// Softmax cross entropy of a linear layer, logits not kept: products of rows with epilogues of their own.  One source file per
// operand mode instantiates them.
//
//   stats   tiles of z = H W + b leave a maximum, a sum of exponentials above it and the label's z for each row and tile of columns
//   grads   tiles of z become P = g (exp(z - lse) - [class == label]), stored in the operands' type, and column sums of it
//   rows    dH (+)= P W^T
#pragma once
#include "grouped.h"

namespace sagnn {

enum XentMode { kXentStats, kXentGrads, kXentRows };

struct XentArgs {
  const void* X; int64_t ldx;                // rows x sum
  const void* W; int64_t ldw;                // sum x cols, or cols x sum
  int64_t m;                                 // rows at most
  const int32_t* count;                      // how many there are, on the device; NULL: m
  int32_t cols, sum, run, mode;
  int32_t col_tiles; int64_t first;          // of the launch
  // stats, grads
  const float* bias; const int32_t* labels;  // bias of the first column on, or NULL
  int32_t class0, classes;                   // class of the first column, all classes
  float2* stats; float* z_label;             // col_tiles x m; m.  Or, with one tile of columns, NULL and
  float* loss; float* lse;                   // the results
  // grads; the rows are `map`'s
  const int32_t* map; const float* row_lse; const float* grad; float grad_all;
  void* P; int64_t ldp; int32_t stored;      // columns that are stored, zeros behind `cols`
  float* bias_parts;                         // row tiles x cols, or NULL
  // rows
  float* sums; bool add, last;               // between pieces of the classes: m x cols
  void* out; int64_t ldo;                    // rows by `map`
};

// LDS of the epilogues: maxima, sums and the label's z of every row; sums of every column
constexpr int xent_lds(int wm, int wn, int tm, int tn) {
  const int rows = wm * tm * 32 * (wn * 8 + 4), cols = wn * tn * 32 * wm * 8;
  return rows > cols ? rows : cols;
}

// The products of grouped.h, grouped_direct.h and grouped_staged.h by one name
template <typename S_, int PREC, bool TRB, int WM_, int WN_, int TM_, int TN_, int BK, bool LONG>
struct SmallProduct {
  using S = S_;
  static constexpr int WM = WM_, WN = WN_, TM = TM_, TN = TN_, kThreads = WM * WN * 64;
  static constexpr int kOperands = TileShape<PREC, false, WM * TM * 32, BK>::kBytes + TileShape<PREC, TRB, WN * TN * 32, BK>::kBytes;
  static constexpr int kLds = kOperands > xent_lds(WM, WN, TM, TN) ? kOperands : xent_lds(WM, WN, TM, TN);
  static constexpr bool kTransW = !TRB;
  static __device__ __forceinline__ void run(const S* A, int64_t lda, int rows, const S* B, int64_t ldb, int cols, int64_t sum, char* smem,
                                             floatx16 (&acc)[TM][TN], int32_t run) {
    tile_product<S, PREC, false, TRB, WM, WN, TM, TN, BK, LONG>(A, lda, rows, B, ldb, cols, sum, smem, acc, run);
  }
};

// Class weights of e^x: x log2(e) is rounded, so the result is good to (1 + |x|) 2^-23
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

// z = acc + bias in place, -inf behind the last column
template <typename C>
__device__ __forceinline__ void add_bias(const XentArgs& a, int64_t c0, int cols, floatx16 (&acc)[C::TM][C::TN], float behind) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int tn = 0; tn < C::TN; ++tn)
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int c = ((wave % C::WN) * C::TN + tn) * 32 + 8 * (v / 4) + 4 * (lane >> 5) + v % 4;
      const bool in = c < cols;
      const float b = a.bias && in ? a.bias[c0 + c] : 0.f;
#pragma unroll
      for (int tm = 0; tm < C::TM; ++tm) acc[tm][tn][v] = in ? acc[tm][tn][v] + b : behind;
    }
}

template <typename C>
__device__ __forceinline__ void xent_stats(const XentArgs& a, int64_t r0, int32_t col, int64_t c0, int rows, int cols, char* smem,
                                           floatx16 (&acc)[C::TM][C::TN]) {
  constexpr int BM = C::WM * C::TM * 32;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  add_bias<C>(a, c0, cols, acc, -INFINITY);
  float2* place = reinterpret_cast<float2*>(smem);           // [WN][BM]
  float* z_label = reinterpret_cast<float*>(place + C::WN * BM);
#pragma unroll
  for (int tm = 0; tm < C::TM; ++tm) {
    const int r = ((wave / C::WN) * C::TM + tm) * 32 + (lane & 31);
    const int64_t label = (r < rows ? (int64_t)a.labels[r0 + r] : -1) - c0;          // column of this tile, or outside it
    float most = -INFINITY;
#pragma unroll
    for (int tn = 0; tn < C::TN; ++tn)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int c = ((wave % C::WN) * C::TN + tn) * 32 + 8 * (v / 4) + 4 * (lane >> 5) + v % 4;
        most = fmaxf(most, acc[tm][tn][v]);
        if (c == label && c < cols) {
          if (a.stats) a.z_label[r0 + r] = acc[tm][tn][v];
          else z_label[r] = acc[tm][tn][v];
        }
      }
    most = fmaxf(most, __shfl_xor(most, 32));
    const float s = shift_of(most);
    float sum = 0.f;
#pragma unroll
    for (int tn = 0; tn < C::TN; ++tn)
#pragma unroll
      for (int v = 0; v < 16; ++v) sum += exp_of(acc[tm][tn][v] - s);
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

template <typename C>
__device__ __forceinline__ void xent_grads(const XentArgs& a, int64_t r0, int64_t row_tile, int64_t c0, int rows, int cols, char* smem,
                                           floatx16 (&acc)[C::TM][C::TN]) {
  constexpr int BN = C::WN * C::TN * 32;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  add_bias<C>(a, c0, cols, acc, -INFINITY);
#pragma unroll
  for (int tm = 0; tm < C::TM; ++tm) {
    const int r = ((wave / C::WN) * C::TM + tm) * 32 + (lane & 31);
    const bool in = r < rows;
    const int64_t row = in ? a.map[r0 + r] : 0;
    const float lse = in ? a.row_lse[row] : 0.f, g = in ? a.grad_all * (a.grad ? a.grad[row] : 1.f) : 0.f;
    const int64_t label = in ? (int64_t)a.labels[row] - a.class0 - c0 : -1;
#pragma unroll
    for (int tn = 0; tn < C::TN; ++tn)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int c = ((wave % C::WN) * C::TN + tn) * 32 + 8 * (v / 4) + 4 * (lane >> 5) + v % 4;
        const float p = exp_of(acc[tm][tn][v] - lse) - (c == label ? 1.f : 0.f);
        acc[tm][tn][v] = in && c < cols ? p * g : 0.f;
      }
  }
  if (a.bias_parts) {                             // sums over the rows, of what is not rounded yet
    float* place = reinterpret_cast<float*>(smem);           // [WM][2][BN]
#pragma unroll
    for (int tn = 0; tn < C::TN; ++tn)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        float x = 0.f;
#pragma unroll
        for (int tm = 0; tm < C::TM; ++tm) x += acc[tm][tn][v];
        x = sixteen_sum(x);
        if ((lane & 15) == 0)
          place[((wave / C::WN) * 2 + ((lane >> 4) & 1)) * BN + ((wave % C::WN) * C::TN + tn) * 32 + 8 * (v / 4) + 4 * (lane >> 5) + v % 4] = x;
      }
    __syncthreads();
    for (int c = threadIdx.x; c < cols; c += C::kThreads) {
      float x = 0.f;
#pragma unroll
      for (int w = 0; w < 2 * C::WM; ++w) x += place[w * BN + c];
      a.bias_parts[row_tile * a.cols + c0 + c] = x;
    }
    __syncthreads();
  }
  using S = typename C::S;
  S* P = reinterpret_cast<S*>(a.P) + r0 * a.ldp + c0;
  const int stored = a.stored - c0 < BN ? (int)(a.stored - c0) : BN;
  tile_fours<C::WM, C::WN, C::TM, C::TN>(acc, [&](int r, int c, float (&y)[4]) {
    if (r < rows) store_four(P + (int64_t)r * a.ldp + c, y, stored - c);
  });
}

template <typename C>
__device__ __forceinline__ void xent_rows(const XentArgs& a, int64_t r0, int64_t c0, int rows, int cols, floatx16 (&acc)[C::TM][C::TN]) {
  using S = typename C::S;
  float* sums = a.sums + r0 * a.cols + c0;
  S* out = reinterpret_cast<S*>(a.out) + c0;
  tile_fours<C::WM, C::WN, C::TM, C::TN>(acc, [&](int r, int c, float (&y)[4]) {
    if (r >= rows) return;
    if (a.add)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (c + i < cols) y[i] += sums[(int64_t)r * a.cols + c + i];
    if (a.last) store_four(out + (int64_t)a.map[r0 + r] * a.ldo + c, y, cols - c);
    else store_four(sums + (int64_t)r * a.cols + c, y, cols - c);
  });
}

// Tiles in bands of eight rows of them, rows fastest, so that the tiles that an XCD has at a time share both operands' rows
constexpr int kXentBand = 8;
template <typename C>
__global__ __launch_bounds__(C::kThreads) void xent_kernel(const XentArgs a) {
  constexpr int BM = C::WM * C::TM * 32, BN = C::WN * C::TN * 32;
  __shared__ __attribute__((aligned(1024))) char smem[C::kLds];
  const int64_t m = a.count ? (*a.count < 0 ? 0 : *a.count > a.m ? a.m : *a.count) : a.m;
  const int32_t row_tiles = (int32_t)((m + BM - 1) / BM);
  const int64_t block = a.first + blockIdx.x, total = (int64_t)row_tiles * a.col_tiles;
  if (block >= total) return;
  const int32_t id = xcd_run((int32_t)block, (int32_t)total), band = id / (kXentBand * a.col_tiles), in = id - band * kXentBand * a.col_tiles;
  const int32_t high = row_tiles - band * kXentBand < kXentBand ? row_tiles - band * kXentBand : kXentBand;
  const int32_t row = band * kXentBand + in % high, col = in / high;
  const int64_t r0 = (int64_t)row * BM, c0 = (int64_t)col * BN;
  const int rows = (int)(m - r0 < BM ? m - r0 : BM), cols = (int)(a.cols - c0 < BN ? a.cols - c0 : BN);
  using S = typename C::S;
  floatx16 acc[C::TM][C::TN];
  C::run(reinterpret_cast<const S*>(a.X) + r0 * a.ldx, a.ldx, rows, reinterpret_cast<const S*>(a.W) + c0 * (C::kTransW ? a.ldw : 1), a.ldw, cols, a.sum,
         smem, acc, a.run);
  __syncthreads();
  if (a.mode == kXentStats) xent_stats<C>(a, r0, col, c0, rows, cols, smem, acc);
  else if (a.mode == kXentGrads) xent_grads<C>(a, r0, row, c0, rows, cols, smem, acc);
  else xent_rows<C>(a, r0, c0, rows, cols, acc);
}

#define SAGNN_XENT_MODE(name) int xent_##name(const XentArgs& a, int tile, bool trans_w, hipStream_t s);
SAGNN_XENT_MODE(fp32)
SAGNN_XENT_MODE(fp32_bf16)
SAGNN_XENT_MODE(fp32_bf16x3)
SAGNN_XENT_MODE(bf16)
#undef SAGNN_XENT_MODE

template <typename C>
int xent_launch(const XentArgs& args, hipStream_t s) {
  const int64_t blocks = ceil_div(args.m, C::WM * C::TM * 32) * args.col_tiles, most = most_blocks(C::kThreads) / 8 * 8;
  XentArgs a = args;
  for (a.first = 0; a.first < blocks; a.first += most) {
    xent_kernel<C><<<dim3((uint32_t)(blocks - a.first < most ? blocks - a.first : most)), C::kThreads, 0, s>>>(a);
    SAGNN_LAUNCH_CHECK();
  }
  return SAGNN_OK;
}
template <typename S, int PREC, int BK, bool TRB, bool LONG>
int xent_small_as(const XentArgs& a, int tile, hipStream_t s) {
  if (tile == kTile128) return xent_launch<SmallProduct<S, PREC, TRB, 2, 2, 2, 2, BK, LONG>>(a, s);
  if (tile == kTile128x64) return xent_launch<SmallProduct<S, PREC, TRB, 2, 2, 2, 1, BK, LONG>>(a, s);
  return xent_launch<SmallProduct<S, PREC, TRB, 1, 4, 1, 1, BK, LONG>>(a, s);
}
template <typename S, int PREC, int BK>
int xent_small(const XentArgs& a, int tile, bool trans_w, hipStream_t s) {
  const bool several = a.sum > a.run;
  if (trans_w) return several ? xent_small_as<S, PREC, BK, false, true>(a, tile, s) : xent_small_as<S, PREC, BK, false, false>(a, tile, s);
  return several ? xent_small_as<S, PREC, BK, true, true>(a, tile, s) : xent_small_as<S, PREC, BK, true, false>(a, tile, s);
}

}  // namespace sagnn
