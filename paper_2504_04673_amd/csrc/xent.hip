// Softmax cross entropy over the classes of a linear layer: entry points, plans, and what stands between the products of xent.h.
//
// Forward, tiles of the logits live in registers: each leaves a maximum and a sum for each of its rows, and a second launch joins a row's.
// Backward the classes are cut into pieces.  A piece's logits are multiplied anew, become P = g (softmax - one-hot) in the epilogue and are stored
// in the operands' type; dH takes P W^T of piece after piece, dW and the bias's gradient are the piece's own.  2 m k n operations forward
// and 6 backward, of which 2 are the price of a memory of one piece.
// Rows without a label are no part of the gradients: a vertex in three has one, often one in a hundred.  Those with one are listed first and their
// features copied (where all have one, taken as they lie), so that the products are as long as the list, and a NaN in a row that has none meets nothing.
//
// Bound by the matrix cores where features are wide: 8192 x 1024 x 131072 bfloat16 forward 2.1 ms (1040 TFLOP/s), a step 8.2 to 8.3 ms, 1060 TFLOP/s of what
// is multiplied; with narrow features by the epilogues' vector instructions, in three terms by the conversion: 170 k x 128 x 172, two in five labelled, 262 us.
#include <initializer_list>
#include <type_traits>

#include "rows.h"
#include "xent.h"

namespace sagnn {
namespace {

constexpr int kListBlocks = 1024;                 // of rows, at most (each reads all their counts)
constexpr int kListThreads = 256;
constexpr int kListFew = 4096;                    // rows whose labels every block counts itself, a launch less
// Bytes of P at a time, about, and classes of a piece: dH's sums are read and written once for each piece, and dW's tiles have to be enough for the chip
// (8192 x 1024 x 131072 bfloat16: pieces of 4096 classes 10.8 ms, 8192 13.0, 16384 9.04, 32768 8.78, 65536 8.6 to 8.9)
constexpr int64_t kPieceBytes = int64_t(512) << 20;
constexpr int32_t kPieceLeast = 1024, kPieceMost = 32768;
constexpr int64_t kLeastBytes = int64_t(4) << 30;   // of P in pieces of kPieceLeast; beyond that, tens of millions of rows, they are narrower
// Pieces at most: dH's sums are added over them in turn, in 32 bits
constexpr int32_t kPiecesMost = 384;
// Rows up to which a bfloat16 P is kept in two terms, the value and what its rounding leaves, each of them a row of dH's and dW's products: they meet 2^-16 of P,
// not 2^-8.  Of more rows those roundings add to the results' own as errors of other sign (1.05 to 1.3 times in the norm, 2000 to 2 classes); of few one of them decides (a row's
// label outweighs its other classes), and the gradients were up to three times as far off as by their own rounding.  The weights' bytes bound these products where rows are few
// (a step, with one term and with two: 1 x 256 x 50000 72 and 77 us, 16 x 1024 x 131072 343 and 358, 128 x 4096 x 131072 1395 and 1675, 512 x 256 x 32768 112 and 148).
// Beyond that weights of the rows are no part of P: equal ones would round most labels' terms alike and shift all gradients by up to 2^-8 (3000 x 256 x 2000, weights of 1 + 2^-8:
// 0.0040 against 64 bits, the results' own rounding being 0.0017, 0.0017 this way; random weights 0.0022 and 0.0017).  dH's rows are multiplied by them
// afterwards; dW sums over the rows, so that they are on the other operand, two terms of weighted H beside each other in twice the columns (a step with weights,
// in P and this way: 2 M x 128 x 47 970 and 1380 us, 170 k x 128 x 172 168 and 193, 8192 x 128 x 65536 1610 and 1727, 8192 x 1024 x 131072 8.05 and 10.5 ms).
constexpr int64_t kTwoTerms = 512, kTwoTermsWeighted = 1024;
// Bytes of the sums of dH's shares
constexpr int64_t kSumBytes = int64_t(512) << 20;

__device__ __forceinline__ bool known(int32_t label, int32_t classes) { return label >= 0 && label < classes; }

// Rows with a label in each block of `each` rows
__global__ __launch_bounds__(kListThreads) void label_count_kernel(const int32_t* __restrict__ labels, int64_t m, int64_t each, int32_t classes,
                                                                   int32_t* __restrict__ counts) {
  __shared__ int32_t room[kListThreads / 64];
  const int64_t end = (blockIdx.x + 1) * each < m ? (blockIdx.x + 1) * each : m;
  int32_t n = 0;
  for (int64_t r = blockIdx.x * each + threadIdx.x; r < end; r += kListThreads) n += known(labels[r], classes);
  for (int d = 1; d < 64; d *= 2) n += __shfl_xor(n, d);
  if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = n;
  __syncthreads();
  if (threadIdx.x == 0) counts[blockIdx.x] = room[0] + room[1] + room[2] + room[3];
}

// map[i] = row of the i-th label; H's rows one behind the other in rows of ldc values (zeros behind the k there are), unless every row has one and
// `needed` is not set: then H itself will do; each as often as P has terms; zeros in dH's rows without one, and in `clear`.  bounds = {0, how many, 0, how many
// rows of terms}.  counts NULL: few rows, whose labels each block counts itself.  `weighted`, if so: the rows, rounded to bfloat16 as the products
// take them, times `weights`, each in two bfloat16 terms of ldc values beside each other.
template <typename T, bool WEIGHTED>
__global__ __launch_bounds__(kListThreads) void label_list_kernel(const int32_t* __restrict__ labels, int64_t m, int64_t each, int32_t classes,
                                                                  const int32_t* __restrict__ counts, int32_t* __restrict__ map, int32_t* __restrict__ bounds,
                                                                  const T* __restrict__ H, int64_t ldh, int32_t k, T* __restrict__ rows, int64_t ldc, int terms,
                                                                  T* __restrict__ dH, int64_t lddh, int lanes, bool needed, float* __restrict__ clear,
                                                                  int32_t n_clear, const float* __restrict__ weights, T* __restrict__ weighted) {
  __shared__ int32_t room[kListThreads / 64];
  __shared__ int32_t place[kListThreads];          // of a row of the round: its number in the list, or -1
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int32_t before = 0, every = 0;                   // before this block; all
  if (counts) {
    for (int b = threadIdx.x; b < (int)gridDim.x; b += kListThreads) {
      const int32_t n = counts[b];
      every += n;
      before += b < (int)blockIdx.x ? n : 0;
    }
  } else {
    for (int r = threadIdx.x; r < (int)m; r += kListThreads) {
      const int32_t n = known(labels[r], classes);
      every += n;
      before += r < (int)blockIdx.x * (int)each ? n : 0;
    }
  }
  if (clear)
    for (int64_t i = (int64_t)blockIdx.x * kListThreads + threadIdx.x; i < n_clear; i += (int64_t)gridDim.x * kListThreads) clear[i] = 0.f;
  for (int d = 1; d < 64; d *= 2) {
    before += __shfl_xor(before, d);
    every += __shfl_xor(every, d);
  }
  if (lane == 0) {
    room[wave] = before;
    place[wave] = every;
  }
  __syncthreads();
  before = room[0] + room[1] + room[2] + room[3];
  every = place[0] + place[1] + place[2] + place[3];
  const int64_t end = (blockIdx.x + 1) * each < m ? (blockIdx.x + 1) * each : m;
  for (int64_t r0 = blockIdx.x * each; r0 < end; r0 += kListThreads) {
    const int64_t r = r0 + threadIdx.x;
    const bool in = r < end && known(labels[r], classes);
    const uint64_t all = __ballot(in);
    __syncthreads();
    if (lane == 0) room[wave] = __popcll(all);
    __syncthreads();
    int32_t at = before + __popcll(all & ((1ull << lane) - 1));
    for (int w = 0; w < wave; ++w) at += room[w];
    place[threadIdx.x] = in ? at : -1;
    if (in) map[at] = (int32_t)r;
    before += room[0] + room[1] + room[2] + room[3];
    __syncthreads();
    // `lanes` of them to a row
    const int n = end - r0 < kListThreads ? (int)(end - r0) : kListThreads, own = threadIdx.x & (lanes - 1);
    for (int i = threadIdx.x / lanes; i < n; i += kListThreads / lanes) {
      const int32_t to = place[i];
      const bool copied = needed || every != m;
      if (to >= 0 && !copied && !WEIGHTED) break;
      if (to >= 0) {
        float g = 1.f;
        if constexpr (WEIGHTED) g = weights[r0 + i];
        for (int c = own * 8; c < ldc; c += lanes * 8) {
          const auto w = load_eight(H + (r0 + i) * ldh + c, k - c, k);
          if (copied)
            for (int e = 0; e < terms; ++e) *reinterpret_cast<TightRun<T, 8>*>(rows + ((int64_t)to * terms + e) * ldc + c) = w;
          if constexpr (WEIGHTED) {
            TightRun<T, 8> high, low;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float x = (float)(__bf16)w.x[e] * g;
              high.x[e] = (T)(__bf16)x;
              low.x[e] = (T)rest_of(x);
            }
            T* to_w = weighted + (int64_t)to * 2 * ldc + c;
            *reinterpret_cast<TightRun<T, 8>*>(to_w) = high;
            *reinterpret_cast<TightRun<T, 8>*>(to_w + ldc) = low;
          }
        }
      }
      else if (dH)
        for (int c = own * 8; c < k; c += lanes * 8) store_eight(dH + (r0 + i) * lddh + c, {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, k - c);
    }
  }
  if (blockIdx.x == gridDim.x - 1 && threadIdx.x == 0) {
    bounds[0] = 0;
    bounds[1] = before;
    bounds[2] = 0;
    bounds[3] = before * terms;
  }
}

// lse and loss of a row from its tiles of columns: 2^log_rows rows a workgroup, its other threads share their tiles, eight at a time.  Sums in 64 bits, and what moves
// them to a new maximum too: there may be half a million tiles, and what their sum loses every class's gradient has (16.7 M classes below a larger one, in chains of
// 32 bits: 1.3e-4).
__device__ __forceinline__ double moved_sum(double sum, float from, float to) {
  return sum == 0. || from == to ? sum : sum * exp((double)shift_of(from) - (double)shift_of(to));
}
__global__ __launch_bounds__(256) void xent_join_kernel(const float2* __restrict__ stats, const float* __restrict__ z_label, int64_t m, int32_t tiles,
                                                        const int32_t* __restrict__ labels, int32_t classes, int log_rows, float* __restrict__ loss,
                                                        float* __restrict__ lse) {
  __shared__ float top[256];
  __shared__ double room[256];
  const int rows = 1 << log_rows, own = threadIdx.x & (rows - 1), shares = 256 >> log_rows, first = threadIdx.x >> log_rows;
  const int64_t r = ((int64_t)blockIdx.x << log_rows) + own;
  float most = -INFINITY;
  double sum = 0.;
  if (r < m)
    for (int t = first; t < tiles; t += 8 * shares) {
      float2 p[8];
      float up = most;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[i] = t + i * shares < tiles ? stats[(t + i * shares) * m + r] : make_float2(-INFINITY, 0.f);
        up = fmaxf(up, p[i].x);
      }
      sum = moved_sum(sum, most, up);
      most = up;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += p[i].y == 0.f ? 0. : (double)p[i].y * (double)exp_of(shift_of(p[i].x) - shift_of(most));
    }
  float up = most;
  top[threadIdx.x] = most;
  __syncthreads();
  for (int half = shares / 2; half > 0; half /= 2) {
    if (first < half) top[threadIdx.x] = up = fmaxf(up, top[threadIdx.x + half * rows]);
    __syncthreads();
  }
  up = top[own];
  room[threadIdx.x] = sum = moved_sum(sum, most, up);
  __syncthreads();
  for (int half = shares / 2; half > 0; half /= 2) {
    if (first < half) room[threadIdx.x] = sum += room[threadIdx.x + half * rows];
    __syncthreads();
  }
  if (threadIdx.x >= rows || r >= m) return;
  const float l = shift_of(up) + logf((float)sum);
  lse[r] = l;
  loss[r] = known(labels[r], classes) ? l - z_label[r] : 0.f;
}

// The bias's gradient: sums over the row tiles, in 64 bits: sixteen columns a workgroup, 64 threads to each where there are many (2 M rows of 47 classes: 43 us,
// with sixteen 103)
template <int kBiasThreads>
__global__ __launch_bounds__(kBiasThreads) void xent_bias_kernel(const float* __restrict__ parts, const int32_t* __restrict__ bounds, int32_t tile_rows,
                                                                 int32_t cols, float* __restrict__ dbias) {
  __shared__ double room[kBiasThreads];
  const int c = blockIdx.x * 16 + (threadIdx.x & 15);
  const int32_t tiles = (bounds[1] + tile_rows - 1) / tile_rows;
  double sum = 0.;
  if (c < cols)
#pragma unroll 8
    for (int t = threadIdx.x >> 4; t < tiles; t += kBiasThreads / 16) sum += (double)parts[(int64_t)t * cols + c];
  room[threadIdx.x] = sum;
  __syncthreads();
  if constexpr (kBiasThreads > 256) {
    if (threadIdx.x < 256) {
#pragma unroll
      for (int p = 1; p < kBiasThreads / 256; ++p) sum += room[p * 256 + threadIdx.x];
      room[threadIdx.x] = sum;
    }
    __syncthreads();
  }
  if (threadIdx.x < 16 && c < cols) {
#pragma unroll
    for (int p = 1; p < 16; ++p) sum += room[p * 16 + threadIdx.x];
    dbias[c] = (float)sum;
  }
}

// dH's listed rows: the sum of the shares' sums, m rows each, of a row's terms, times its weight (grad, may be NULL)
template <typename T>
__global__ __launch_bounds__(256) void xent_rows_kernel(const float* __restrict__ sums, int32_t splits, int64_t m, int terms, float scale, const float* __restrict__ grad,
                                                        const int32_t* __restrict__ bounds, int32_t k, const int32_t* __restrict__ map, T* __restrict__ dH, int64_t lddh) {
  const int64_t fours = (k + 3) / 4, all = bounds[1] * fours;
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < all; i += gridDim.x * 256ll) {
    const int64_t r = i / fours;
    const int c = (int)(i - r * fours) * 4;
    float y[4] = {0.f, 0.f, 0.f, 0.f};
    const float* from = sums + r * terms * k + c;
    const int32_t parts = splits * terms;
    auto part = [&](int32_t p) { return from + (terms == 2 ? (p >> 1) * m * k + (p & 1) * k : p * m * k); };
    if (c + 4 <= k) {
#pragma unroll 4
      for (int32_t s = 0; s < parts; ++s) {
        float x[4];
        __builtin_memcpy(x, reinterpret_cast<const Four<float>*>(part(s)), 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] += x[e];
      }
    } else {
      for (int32_t s = 0; s < parts; ++s)
#pragma unroll
        for (int e = 0; e < 3; ++e)
          if (c + e < k) y[e] += part(s)[e];
    }
    const int64_t row = map[r];
    const float factor = grad ? scale * grad[row] : scale;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] *= factor;
    store_four(dH + row * lddh + c, y, k - c);
  }
}

// A piece's dW from fp32 into its place, or times the scale where it is (no rows: zeros, whatever that is).  second: how far behind a value the rest of it is that weighted rows' second
// terms make; 0: there is none
template <typename T>
__global__ __launch_bounds__(256) void xent_convert_kernel(const float* from, int64_t ldf, int64_t second, int64_t rows, int32_t cols, float factor,
                                                           const int32_t* __restrict__ bounds, T* to, int64_t ldt) {
  const float scale = bounds[1] > 0 ? factor : 0.f;
  const int64_t fours = (cols + 3) / 4, all = rows * fours;
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < all; i += gridDim.x * 256ll) {
    const int64_t r = i / fours;
    const int c = (int)(i - r * fours) * 4;
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float* x = from + r * ldf + c + e;
      y[e] = c + e < cols ? (second ? x[0] + x[second] : x[0]) * scale : 0.f;
    }
    store_four(to + r * ldt + c, y, cols - c);
  }
}

// ------------------------------------------------------------------------------------------

bool valid(int32_t dtype, int32_t transW, int64_t m, int32_t kdim, int32_t classes, int32_t prec) {
  return (dtype == SAGNN_F32 || (dtype == SAGNN_BF16 && prec == SAGNN_GEMM_FP32)) && prec >= SAGNN_GEMM_FP32 && prec <= SAGNN_GEMM_FP32_BF16X3 &&
         !(transW & ~1) && m >= 0 && m <= INT32_MAX && kdim >= 1 && kdim <= SAGNN_GROUPED_MAX_WIDTH && classes >= 1 && classes <= SAGNN_XENT_MAX_CLASSES &&
         ceil_div(m, 32) * ceil_div(classes, 32) <= INT32_MAX;
}

int32_t products(int32_t dtype, int32_t prec) { return dtype == SAGNN_BF16 ? SAGNN_GEMM_BF16 : prec; }

// Which large tile a product can have besides the small ones: none, one that loads straight into LDS, one staged through registers
enum { kSmallOnly = 0, kDirect = 1, kStaged = 2 };
constexpr int64_t kLargeLd = 1 << 20;             // (offsets inside a tile of 256 rows below 2^31)
bool whole_granules(const void* p, int64_t ld, int64_t width) { return aligned16(p) && ld % 8 == 0 && width % 8 == 0 && ld <= kLargeLd; }

// Tile of a product, m rows by cols, `sum` deep, and shares of the summed index (several only with `room` for sums of their own): what the fullest CU
// multiplies, by the tiles' rates, and what it costs to write and read the shares' sums.
struct TilePick { int tile; int32_t splits, share; };
// What the 256 x 256 tile's epilogue costs, in rows of the summed index: with exponentials in it and one workgroup on a CU more than a plain product's 200
// (a step of 170 k x 128 x 172 in bfloat16 took 205 us with 200, 167 with 300; 8192 x 128 x 65536, which keeps the tile, 1594; with 400, without it, 1660).
constexpr double kDirectEnds = 300;
// joined: several tiles of columns cost a launch more.  (The staged tiles' rates 0.8 and 1.4 times as high: 170 k x 128 x 172 in three terms 308 and 267 us
// for 266, 4099 x 200 x 54321 2.67 and 2.92 ms for 2.67.)
TilePick pick_tile(int32_t dtype, int32_t prec, int ways, int64_t m, int64_t cols, int64_t sum, int32_t room, bool joined = false) {
  TilePick best{kTile128, 1, (int32_t)sum};
  double least = 1e300;
  // values of a 128 x 128 tile that a CU multiplies in a microsecond (half of the operations), and bytes that the chip moves in one
  const double a_us = (dtype == SAGNN_BF16 ? 740e6 : prec == SAGNN_GEMM_FP32 ? 133e6 : prec == SAGNN_GEMM_BF16 ? 430e6 : 171e6) / 512, bytes_us = 4e6;
  for (int tile : {kTile128, kTile128x64, kTile32x128, kThin, kDirect256, kStaged256x128, kStaged128x256}) {
    TileCost c = tile_cost(dtype, prec, tile);
    if (tile == kDirect256) c.ends = kDirectEnds;
    if (c.rate == 0 || (tile == kDirect256 && ways != kDirect) || ((tile == kStaged256x128 || tile == kStaged128x256) && ways != kStaged)) continue;
    const int64_t h = grouped_tile_rows(tile), w = grouped_tile_cols(tile);
    const int64_t whole = ceil_div(m, h) * ceil_div(cols, w);
    for (int32_t splits = 1; splits <= room && (splits == 1 || whole * splits < 4 * 256); ++splits) {
      const int64_t share = splits == 1 ? sum : (int64_t)round_up((size_t)ceil_div(sum, splits), 64), n = ceil_div(sum, share);
      if (splits > 1 && share < 512) break;
      if (tile == kDirect256 && share > kRunRounded) continue;
      const int64_t tiles = whole * n;
      const double turns = tiles <= 256 ? 1.25 : tiles < 4 * 256 ? (double)ceil_div(tiles, 256) : tiles / 256.;
      const double cost = turns * h * w * (share + c.ends) / c.rate / a_us + (n > 1 ? 12. * n * m * cols / bytes_us + 5. : 0.) + (joined && cols > w ? 5. : 0.);
      if (cost < least) {
        least = cost;
        best = {tile, (int32_t)n, (int32_t)share};
      }
    }
  }
  return best;
}
// Of the logits: H (or the listed rows, whose ends are padded) and W
int logits_ways(int32_t dtype, const void* H, int64_t ldh, int64_t width, const void* W, int64_t ldw, bool transW, int32_t kdim, int32_t classes) {
  if (dtype == SAGNN_F32) return ldh <= kLargeLd && ldw <= kLargeLd ? kStaged : kSmallOnly;
  return kdim <= kRunBf16 && whole_granules(H, ldh, width) && whole_granules(W, ldw, transW ? kdim : classes) ? kDirect : kSmallOnly;
}
// Of dH: P, whose rows are padded, and W the other way
int rows_ways(int32_t dtype, int64_t ldp, const void* W, int64_t ldw, bool transW, int32_t kdim, int32_t classes) {
  if (dtype == SAGNN_F32) return ldp <= kLargeLd && ldw <= kLargeLd ? kStaged : kSmallOnly;
  return whole_granules(W, ldw, transW ? kdim : classes) ? kDirect : kSmallOnly;
}

int launch(const XentArgs& args, int32_t dtype, int32_t prec, const TilePick& pick, bool trans_w, hipStream_t s) {
  XentArgs a = args;
  const int tile = pick.tile;
  a.splits = pick.splits;
  a.share = pick.share;
  a.run = grouped_run(products(dtype, prec), tile == kThin ? ceil_div(a.share, kThinWaves) : a.share);
  a.col_tiles = (int32_t)ceil_div(a.cols, grouped_tile_cols(tile));
  if (dtype == SAGNN_BF16) return xent_bf16(a, tile, trans_w, s);
  return prec == SAGNN_GEMM_FP32 ? xent_fp32(a, tile, trans_w, s) : prec == SAGNN_GEMM_BF16 ? xent_fp32_bf16(a, tile, trans_w, s) : xent_fp32_bf16x3(a, tile, trans_w, s);
}

struct Room {
  size_t off = 0;
  size_t take(size_t bytes) { const size_t o = off; off += round_up(bytes, 256); return o; }
};

struct FwdPlan { TilePick tile; int32_t col_tiles; size_t stats, z_label, total; };
FwdPlan fwd_plan(int32_t dtype, int32_t prec, int ways, int64_t m, int32_t kdim, int32_t classes) {
  FwdPlan p{};
  p.tile = pick_tile(dtype, prec, ways, m, classes, kdim, 1, true);
  p.col_tiles = (int32_t)ceil_div(classes, grouped_tile_cols(p.tile.tile));
  if (p.col_tiles > 1) {
    Room room;
    p.stats = room.take((size_t)m * p.col_tiles * sizeof(float2));
    p.z_label = room.take((size_t)m * sizeof(float));
    p.total = room.off;
  }
  return p;
}

// dW's products have the listed rows' and P's ends in them, zeros, so that bfloat16 ones go straight into LDS whatever the widths are: they end in a place
// of their own anyway
int32_t padded_width(int32_t dtype, int32_t width) { return dtype == SAGNN_BF16 ? (int32_t)round_up((size_t)width, 8) : width; }

// Whether dW (bfloat16) is made by tiles over all rows, rounded where it belongs, or in chunks of rows through fp32, which are joined and converted: by what each
// takes, the first in whole turns of the CUs (microseconds; 0.027 a row of a tile, at the large tile's rate), the second with its bytes and launches.
bool whole_weights(int32_t dtype, int64_t m, int32_t kdim, int32_t classes) {
  const int64_t tiles = ceil_div(kdim, 256) * ceil_div(classes, 256);
  if (dtype != SAGNN_BF16 || m > kRunRounded || tiles > INT32_MAX) return false;
  const double one = .027 * (m + 200);
  return one * ceil_div(tiles, 256) <= one * tiles / 256. + 12. + 12. * kdim * classes / 4e6;
}

struct BwdPlan {
  int32_t terms;                             // of P
  bool outside;                              // the rows' weights are no part of P: dH's rows are multiplied by them, and dW's product takes weighted rows of H
  int32_t piece, pieces;                     // classes of a piece
  int32_t splits;                            // shares of them that there is room for in dH's sums
  int64_t ldp, ldc;                          // of P, of the listed rows
  size_t map, bounds, counts, rows, weighted, P, sums, weights, parts, bias, weights_bytes, parts_bytes, total;
};
int32_t terms_of(int32_t dtype, int64_t m, bool weighted) { return dtype == SAGNN_BF16 && m <= (weighted ? kTwoTermsWeighted : kTwoTerms) ? 2 : 1; }
BwdPlan bwd_plan(int32_t dtype, int32_t prec, bool weighted, int64_t m, int32_t kdim, int32_t classes) {
  BwdPlan p{};
  p.terms = terms_of(dtype, m, weighted);
  p.outside = weighted && p.terms == 1 && products(dtype, prec) == SAGNN_GEMM_BF16;
  const int64_t size = dtype == SAGNN_BF16 ? 2 : 4, rows = m > 0 ? m : 1;
  int64_t most = kPieceBytes / (rows * size) / 256 * 256;
  const int32_t least = rows * size * kPieceLeast <= kLeastBytes ? kPieceLeast : 256;
  most = most < least ? least : most > kPieceMost ? kPieceMost : most;
  if (most < ceil_div(classes, kPiecesMost)) most = ceil_div(classes, kPiecesMost);
  p.pieces = (int32_t)ceil_div(classes, most);
  p.piece = p.pieces == 1 ? classes : (int32_t)round_up((size_t)ceil_div(classes, p.pieces), 256);
  p.pieces = (int32_t)ceil_div(classes, p.piece);
  p.ldp = (int64_t)round_up((size_t)p.piece, 8);
  p.ldc = (int64_t)round_up((size_t)kdim, 8);
  // dW's products, in either order, of a whole piece and of the last (which may be cut into more parts)
  const int32_t kw = p.outside ? (int32_t)(2 * p.ldc) : padded_width(dtype, kdim);
  const int32_t last = classes - (p.pieces - 1) * p.piece;
  for (int32_t n : {p.piece, last}) {
    if (!p.outside && whole_weights(dtype, m * p.terms, kdim, n)) continue;
    p.weights_bytes = (size_t)padded_width(dtype, p.piece) * kw * 4;
    const size_t one = grouped_weights_bytes(m * p.terms, kw, padded_width(dtype, n)), two = grouped_weights_bytes(m * p.terms, padded_width(dtype, n), kw);
    p.parts_bytes = one > p.parts_bytes ? one : p.parts_bytes;
    p.parts_bytes = two > p.parts_bytes ? two : p.parts_bytes;
    if (last == p.piece) break;
  }
  Room room;
  p.map = room.take((size_t)rows * 4);
  p.bounds = room.take(16);
  p.counts = room.take(kListBlocks * 4);
  p.rows = room.take((size_t)rows * p.terms * p.ldc * size);
  p.weighted = room.take(p.outside ? (size_t)rows * 2 * p.ldc * size : 0);
  p.P = room.take((size_t)rows * p.terms * p.ldp * size);
  // dH's sums: of every share of a piece's classes
  const int64_t share = rows * p.terms * kdim * 4;
  p.splits = share > 0 ? (int32_t)(kSumBytes / share < 1 ? 1 : kSumBytes / share > 32 ? 32 : kSumBytes / share) : 1;
  int32_t splits = 1;
  for (int ways : {kSmallOnly, dtype == SAGNN_BF16 ? kDirect : kStaged}) {
    const int32_t n = pick_tile(dtype, prec, ways, m * p.terms, kdim, p.piece, p.splits).splits;
    if (n > splits) splits = n;
  }
  p.sums = room.take(p.pieces > 1 || splits > 1 || p.terms > 1 ? (size_t)splits * share : 0);
  p.weights = room.take(p.weights_bytes);
  p.parts = room.take(p.parts_bytes);
  p.bias = room.take((size_t)ceil_div(rows, 32) * p.piece * 4);
  p.total = room.off;
  return p;
}

template <typename T>
int list_labels(const BwdPlan& p, char* ws, const int32_t* labels, int64_t m, int32_t classes, const void* H, int64_t ldh, int32_t k, void* dH, int64_t lddh,
                bool needed, float* clear, int32_t n_clear, const float* weights, hipStream_t s) {
  // (many small blocks: 8192 rows of 1024 in blocks of 256 took 429 us)
  int64_t each = ceil_div(m, kListBlocks);
  if (each < 16) each = 16;
  int lanes = 2;
  while (lanes < 64 && lanes * 8 < p.ldc) lanes *= 2;
  const uint32_t blocks = (uint32_t)ceil_div(m > 0 ? m : 1, each);
  int32_t *counts = (int32_t*)(ws + p.counts), *map = (int32_t*)(ws + p.map), *bounds = (int32_t*)(ws + p.bounds);
  if (m <= kListFew) {
    counts = nullptr;
  } else {
    label_count_kernel<<<dim3(blocks), kListThreads, 0, s>>>(labels, m, each, classes, counts);
    SAGNN_LAUNCH_CHECK();
  }
  auto list = [&](auto kernel) {
    kernel<<<dim3(blocks), kListThreads, 0, s>>>(labels, m, each, classes, counts, map, bounds, (const T*)H, ldh, k, (T*)(ws + p.rows), p.ldc, p.terms, (T*)dH, lddh,
                                                 lanes, needed, clear, n_clear, weights, (T*)(ws + p.weighted));
  };
  if (p.outside) list(label_list_kernel<T, true>);
  else list(label_list_kernel<T, false>);
  SAGNN_LAUNCH_CHECK();
  return SAGNN_OK;
}

bool element_aligned(const void* p, int32_t dtype) { return aligned_to(p, dtype == SAGNN_BF16 ? 2 : 4); }
// Two ranges of bytes have nothing in common
bool clear_of(const void* p, size_t bytes_p, const void* q, size_t bytes_q) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return !p || !q || !bytes_p || !bytes_q || a + bytes_p <= b || b + bytes_q <= a;
}
size_t reach(int64_t rows, int64_t ld, int64_t cols, size_t size) { return rows > 0 ? ((size_t)(rows - 1) * ld + cols) * size : 0; }

}  // namespace
}  // namespace sagnn

SAGNN_EXPORT int softmax_xent_workspace_bytes(int32_t dtype, int64_t m, int32_t kdim, int32_t n_classes, int32_t prec, int32_t backward, size_t* bytes) {
  using namespace sagnn;
  if (!bytes || !valid(dtype, 0, m, kdim, n_classes, prec) || (backward & ~1)) return SAGNN_EINVAL;
  if (backward) {
    *bytes = 0;                              // (for either kind of gradient)
    for (int32_t weighted : {0, 1}) {
      size_t b = 0;
      softmax_xent_bwd_workspace_bytes(dtype, m, kdim, n_classes, prec, weighted, &b);
      if (b > *bytes) *bytes = b;
    }
  } else {                                   // (room for any strides and alignments)
    *bytes = 0;
    for (int ways : {kSmallOnly, dtype == SAGNN_BF16 ? kDirect : kStaged}) {
      const size_t b = fwd_plan(dtype, prec, ways, m, kdim, n_classes).total;
      if (b > *bytes) *bytes = b;
    }
  }
  return SAGNN_OK;
}

SAGNN_EXPORT int softmax_xent_bwd_workspace_bytes(int32_t dtype, int64_t m, int32_t kdim, int32_t n_classes, int32_t prec, int32_t weighted, size_t* bytes) {
  using namespace sagnn;
  if (!bytes || !valid(dtype, 0, m, kdim, n_classes, prec) || (weighted & ~1)) return SAGNN_EINVAL;
  *bytes = bwd_plan(dtype, prec, weighted != 0, m, kdim, n_classes).total;
  return SAGNN_OK;
}

SAGNN_EXPORT int softmax_xent_fwd(int32_t dtype, const void* d_H, int64_t ldh, const void* d_W, int64_t ldw, int32_t transW, const float* d_bias,
                                  const int32_t* d_labels, int64_t m, int32_t kdim, int32_t n_classes, int32_t prec, float* d_loss, float* d_lse,
                                  void* d_ws, size_t ws_bytes, void* stream) {
  using namespace sagnn;
  if (!valid(dtype, transW, m, kdim, n_classes, prec) || ldh < kdim || ldw < (transW ? kdim : n_classes)) return SAGNN_EINVAL;
  if (m == 0) return SAGNN_OK;
  if (!d_H || !d_W || !d_labels || !d_loss || !d_lse || !element_aligned(d_H, dtype) || !element_aligned(d_W, dtype) || !aligned_to(d_bias, 4) ||
      !aligned_to(d_labels, 4) || !aligned_to(d_loss, 4) || !aligned_to(d_lse, 4) || !aligned_to(d_ws, 16))
    return SAGNN_EINVAL;
  const size_t size = dtype == SAGNN_BF16 ? 2 : 4, h = reach(m, ldh, kdim, size), w = transW ? reach(n_classes, ldw, kdim, size) : reach(kdim, ldw, n_classes, size);
  for (const float* out : {d_loss, d_lse})
    if (!clear_of(out, m * 4, d_H, h) || !clear_of(out, m * 4, d_W, w) || !clear_of(out, m * 4, d_labels, m * 4) || !clear_of(out, m * 4, d_bias, (size_t)n_classes * 4))
      return SAGNN_EINVAL;
  if (!clear_of(d_loss, m * 4, d_lse, m * 4)) return SAGNN_EINVAL;
  const FwdPlan p = fwd_plan(dtype, prec, logits_ways(dtype, d_H, ldh, kdim, d_W, ldw, transW != 0, kdim, n_classes), m, kdim, n_classes);
  if (p.total > 0 && !d_ws) return SAGNN_EINVAL;
  if (ws_bytes < p.total) return SAGNN_ECAPACITY;
  XentArgs a{};
  a.X = d_H; a.ldx = ldh; a.W = d_W; a.ldw = ldw; a.m = m; a.cols = n_classes; a.sum = a.padded = kdim; a.mode = kXentStats; a.bias = d_bias; a.labels = d_labels;
  a.classes = n_classes; a.loss = d_loss; a.lse = d_lse;
  if (p.total > 0) {
    a.stats = (float2*)((char*)d_ws + p.stats);
    a.z_label = (float*)((char*)d_ws + p.z_label);
  }
  hipStream_t s = (hipStream_t)stream;
  const int rc = launch(a, dtype, prec, p.tile, transW != 0, s);
  if (rc != SAGNN_OK || p.total == 0) return rc;
  // (16 threads to a row of many tiles: 8192 rows of 1024 of them, four threads to each, took 106 us; 64 or more where the tiles are two megabytes or chains long)
  const int log_rows = p.col_tiles <= 16 ? 6 : p.col_tiles <= 1024 && m * p.col_tiles > (1 << 18) ? 4 : m >= 4 ? 2 : 0;
  xent_join_kernel<<<dim3((uint32_t)ceil_div(m, 1 << log_rows)), 256, 0, s>>>(a.stats, a.z_label, m, p.col_tiles, d_labels, n_classes, log_rows, d_loss, d_lse);
  SAGNN_LAUNCH_CHECK();
  return SAGNN_OK;
}

SAGNN_EXPORT int softmax_xent_bwd(int32_t dtype, const void* d_H, int64_t ldh, const void* d_W, int64_t ldw, int32_t transW, const float* d_bias,
                                  const int32_t* d_labels, const float* d_lse, const float* d_grad, double grad_all, int64_t m, int32_t kdim,
                                  int32_t n_classes, int32_t prec, void* d_dH, int64_t lddh, void* d_dW, float* d_dbias, void* d_ws, size_t ws_bytes,
                                  void* stream) {
  using namespace sagnn;
  if (!valid(dtype, transW, m, kdim, n_classes, prec) || ldh < kdim || ldw < (transW ? kdim : n_classes) || (d_dH && lddh < kdim)) return SAGNN_EINVAL;
  if (!d_W || (m > 0 && (!d_H || !d_labels || !d_lse)) || !element_aligned(d_H, dtype) || !element_aligned(d_W, dtype) || !aligned_to(d_bias, 4) ||
      !aligned_to(d_labels, 4) || !aligned_to(d_lse, 4) || !aligned_to(d_grad, 4) || !element_aligned(d_dH, dtype) || !element_aligned(d_dW, dtype) ||
      !aligned_to(d_dbias, 4) || !aligned_to(d_ws, 16))
    return SAGNN_EINVAL;
  const size_t size = dtype == SAGNN_BF16 ? 2 : 4;
  {
    const struct { const void* p; size_t bytes; } in[] = {{d_H, reach(m, ldh, kdim, size)}, {d_W, transW ? reach(n_classes, ldw, kdim, size) : reach(kdim, ldw, n_classes, size)},
                                                          {d_bias, (size_t)n_classes * 4}, {d_labels, (size_t)m * 4}, {d_lse, (size_t)m * 4}, {d_grad, (size_t)m * 4}};
    const struct { const void* p; size_t bytes; } out[] = {{d_dH, reach(m, lddh, kdim, size)}, {d_dW, (size_t)n_classes * kdim * size}, {d_dbias, (size_t)n_classes * 4}};
    for (int o = 0; o < 3; ++o) {
      for (const auto& i : in)
        if (!clear_of(out[o].p, out[o].bytes, i.p, i.bytes)) return SAGNN_EINVAL;
      for (int q = 0; q < o; ++q)
        if (!clear_of(out[o].p, out[o].bytes, out[q].p, out[q].bytes)) return SAGNN_EINVAL;
    }
  }
  const BwdPlan p = bwd_plan(dtype, prec, d_grad != nullptr, m, kdim, n_classes);
  if (!d_ws) return SAGNN_EINVAL;
  if (ws_bytes < p.total) return SAGNN_ECAPACITY;
  char* ws = (char*)d_ws;
  hipStream_t s = (hipStream_t)stream;
  // Where every row has a label H itself is taken, if it lies as well as the copy would (617 k x 1344 of 50 classes, three terms, all labelled: 5.8 ms
  // with the copy).  Only the device knows.
  const bool itself = p.terms == 1 && (dtype == SAGNN_BF16 ? whole_granules(d_H, ldh, kdim) : ldh <= kLargeLd);
  // The bias's gradient of one tile of rows is its sums: written there, over zeros for the case that there is no such row
  auto logits = [&](const void* W, int32_t n) {
    return pick_tile(dtype, prec, logits_ways(dtype, ws + p.rows, p.ldc * p.terms, p.ldc, W, ldw, transW != 0, kdim, n), m, n, kdim, 1);
  };
  const int32_t last = n_classes - (p.pieces - 1) * p.piece;
  const bool direct_bias = d_dbias && m <= grouped_tile_rows(logits(d_W, p.piece).tile) && m <= grouped_tile_rows(logits(d_W, last).tile);
  float* clear = direct_bias ? d_dbias : nullptr;
  int rc = dtype == SAGNN_BF16 ? list_labels<__bf16>(p, ws, d_labels, m, n_classes, d_H, ldh, kdim, d_dH, lddh, !itself, clear, n_classes, d_grad, s)
                               : list_labels<float>(p, ws, d_labels, m, n_classes, d_H, ldh, kdim, d_dH, lddh, !itself, clear, n_classes, d_grad, s);
  const int32_t* bounds = (const int32_t*)(ws + p.bounds);
  const int32_t* term_bounds = bounds + (p.terms == 2 ? 2 : 0);
  const int64_t terms = m * p.terms;
  // A factor of all rows is no part of a P that is rounded to bfloat16, here or on its way into the products: its rounding would be one for most labels'
  // terms and shift all gradients by up to 2^-8
  const bool rounded = products(dtype, prec) == SAGNN_GEMM_BF16;
  const float scale = rounded ? (float)grad_all : 1.f;
  TilePick rows{};
  for (int32_t at = 0; at < n_classes && rc == SAGNN_OK; at += p.piece) {
    const int32_t n = n_classes - at < p.piece ? n_classes - at : p.piece;
    XentArgs a{};
    a.X = ws + p.rows; a.ldx = p.ldc * p.terms; a.W = (const char*)d_W + (size_t)at * (transW ? ldw : 1) * size; a.ldw = ldw; a.m = m; a.count = bounds + 1;
    a.all = itself ? d_H : nullptr; a.ldall = ldh; a.cols = n; a.sum = kdim; a.mode = p.terms == 2 ? kXentTwo : kXentGrads; a.bias = d_bias ? d_bias + at : nullptr; a.labels = d_labels; a.class0 = at; a.classes = n_classes;
    a.map = (const int32_t*)(ws + p.map); a.row_lse = d_lse; a.grad = d_grad; a.outside = p.outside; a.grad_all = rounded ? 1.f : (float)grad_all; a.scale = scale; a.P = ws + p.P; a.ldp = p.ldp;
    a.stored = (int32_t)round_up((size_t)n, 8); a.bias_parts = direct_bias ? d_dbias + at : d_dbias ? (float*)(ws + p.bias) : nullptr;
    a.padded = (int32_t)p.ldc;
    const TilePick tile = logits(a.W, n);
    if (m > 0) rc = launch(a, dtype, prec, tile, transW != 0, s);
    if (rc == SAGNN_OK && d_dbias && !direct_bias) {
      const int32_t high = grouped_tile_rows(tile.tile);
      const dim3 grid((uint32_t)ceil_div(n, 16));
      if (m > 256 * high) xent_bias_kernel<1024><<<grid, 1024, 0, s>>>(a.bias_parts, bounds, high, n, d_dbias + at);
      else xent_bias_kernel<256><<<grid, 256, 0, s>>>(a.bias_parts, bounds, high, n, d_dbias + at);
      SAGNN_LAUNCH_CHECK();
    }
    if (rc == SAGNN_OK && d_dH && m > 0) {
      // (the last piece in as many shares as the others, whose sums it adds to)
      if (at == 0) rows = pick_tile(dtype, prec, rows_ways(dtype, p.ldp, a.W, ldw, transW != 0, kdim, n_classes), terms, kdim, p.piece, p.splits);
      const bool summed = p.pieces > 1 || rows.splits > 1 || p.terms > 1;
      TilePick pick = rows;
      if (pick.splits == 1) pick.share = n;
      XentArgs b{};
      b.X = a.P; b.ldx = p.ldp; b.W = a.W; b.ldw = ldw; b.m = terms; b.count = term_bounds + 1; b.scale = scale; b.cols = kdim; b.sum = n; b.mode = kXentRows; b.map = a.map;
      b.grad = p.outside ? d_grad : nullptr; b.sums = summed ? (float*)(ws + p.sums) : nullptr; b.add = at > 0; b.out = d_dH; b.ldo = lddh;
      b.padded = a.stored; b.wide = aligned16(d_dH) && lddh % 8 == 0 && kdim % 8 == 0;
      rc = launch(b, dtype, prec, pick, transW == 0, s);
      if (rc == SAGNN_OK && summed && at + n == n_classes) {
        const int64_t blocks = ceil_div(m * ceil_div(kdim, 4), 256);
        const dim3 grid((uint32_t)(blocks < 8192 ? blocks : 8192));
        if (dtype == SAGNN_BF16) xent_rows_kernel<__bf16><<<grid, 256, 0, s>>>(b.sums, rows.splits, terms, p.terms, scale, b.grad, bounds, kdim, b.map, (__bf16*)d_dH, lddh);
        else xent_rows_kernel<float><<<grid, 256, 0, s>>>(b.sums, rows.splits, terms, p.terms, scale, b.grad, bounds, kdim, b.map, (float*)d_dH, lddh);
        SAGNN_LAUNCH_CHECK();
      }
    }
    if (rc == SAGNN_OK && d_dW && !p.outside && whole_weights(dtype, terms, kdim, n)) {
      XentWeightArgs w{};
      const void* whole = itself ? d_H : a.X;
      const int64_t ldwhole = itself ? ldh : p.ldc;
      w.scale = scale; w.A = transW ? a.P : a.X; w.lda = transW ? p.ldp : p.ldc; w.A2 = transW ? a.P : whole; w.lda2 = transW ? p.ldp : ldwhole;
      w.B = transW ? a.X : a.P; w.ldb = transW ? p.ldc : p.ldp; w.B2 = transW ? whole : a.P; w.ldb2 = transW ? ldwhole : p.ldp;
      w.count = term_bounds + 1; w.m = terms; w.rows = transW ? n : kdim; w.cols = transW ? kdim : n;
      w.row_tiles = (int32_t)ceil_div(w.rows, 256); w.col_tiles = (int32_t)ceil_div(w.cols, 256);
      w.ldo = transW ? kdim : n_classes; w.out = (__bf16*)d_dW + (size_t)at * (transW ? kdim : 1);
      w.wide = aligned16(w.out) && w.ldo % 8 == 0 && w.cols % 8 == 0;
      rc = xent_weights_bf16(w, s);
    } else if (rc == SAGNN_OK && d_dW) {
      // (fp32 weights whose piece lies in one place are written there)
      const bool there = dtype == SAGNN_F32 && !p.outside && (transW || p.pieces == 1);
      float* dW = there ? (float*)d_dW + (size_t)at * (transW ? kdim : 1) : (float*)(ws + p.weights);
      GroupedArgs w{};
      w.off = term_bounds; w.groups = 1; w.m = terms; w.dW = dW; w.partial = (float*)(ws + p.parts);
      // (weighted rows: their two terms are the first and the second half of one operand's columns, and dW their products' sum)
      const int32_t kw = p.outside ? (int32_t)(2 * p.ldc) : padded_width(dtype, kdim), nw = padded_width(dtype, n);
      const void* rows_of_h = p.outside ? ws + p.weighted : a.X;
      const int64_t ldr = p.outside ? 2 * p.ldc : p.ldc;
      w.X = transW ? a.P : rows_of_h; w.ldx = transW ? p.ldp : ldr; w.kdim = transW ? nw : kw;
      w.G = transW ? rows_of_h : a.P; w.ldg = transW ? ldr : p.ldp; w.nout = transW ? kw : nw;
      if (itself && !p.outside) {
        w.listed = bounds + 1;
        w.X2 = transW ? a.P : d_H; w.ldx2 = transW ? p.ldp : ldh;
        w.G2 = transW ? d_H : a.P; w.ldg2 = transW ? ldh : p.ldp;
      }
      rc = grouped_weights(w, dtype, prec, s);
      if (rc == SAGNN_OK && (!there || scale != 1.f)) {
        const int64_t rows = transW ? n : kdim, ldt = transW ? kdim : n_classes;
        const int32_t cols = transW ? kdim : n;
        const int64_t blocks = ceil_div(rows * ceil_div(cols, 4), 256);
        const dim3 grid((uint32_t)(blocks < 4096 ? blocks : 4096));
        const size_t first = (size_t)at * (transW ? kdim : 1);
        const int64_t second = !p.outside ? 0 : transW ? p.ldc : p.ldc * (int64_t)w.nout;
        if (dtype == SAGNN_BF16) xent_convert_kernel<__bf16><<<grid, 256, 0, s>>>(dW, w.nout, second, rows, cols, scale, bounds, (__bf16*)d_dW + first, ldt);
        else xent_convert_kernel<float><<<grid, 256, 0, s>>>(dW, w.nout, second, rows, cols, scale, bounds, (float*)d_dW + first, ldt);
        SAGNN_LAUNCH_CHECK();
      }
    }
  }
  return rc;
}
