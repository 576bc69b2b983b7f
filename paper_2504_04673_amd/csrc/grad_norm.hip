// The 2-norm over all gradient tensors of a model, and the tensors scaled so that it does not exceed a bound.
#include <algorithm>
#include <cmath>
#include <new>

#include "common.h"

namespace sagnn {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxBlocks = 1024;     // workgroups of a launch that sums, and the sums that it leaves
constexpr int kListBytes = 3840;     // of a launch's arguments (4 KB at most), in which the tensors travel
// Values that a workgroup takes at a time: so many that kMaxBlocks workgroups have one each, within these bounds.  (More
// workgroups are more sums for each of them to join: 2 x 10 M values, 2048 workgroups 8.5 us to sum and 16.7 to scale, 1024 8.9 and
// 14.7, 512 10.1 and 14.1; half a billion 188 and 361, 186 and 358, 212 and 352.)
constexpr int kLeastPiece = 2048, kMostPiece = 16384;

// Tensors of one launch.  Addresses have 48 bits and a tensor's end 15, so that a launch takes 318 tensors, or 212 with places for
// results (211 tensors as 24 bytes each, two launches to sum and two to scale: 51 us in place of 41).
template <bool OUT>
struct List {
  static constexpr int kMost = (kListBytes - 16) / (OUT ? 18 : 12), kAddresses = OUT ? 2 * kMost : kMost;
  int32_t first[kMost + 1];          // pieces before the tensor
  uint32_t low[kAddresses];          // of the tensors, then of their results
  uint16_t high[kAddresses];
  uint16_t end[kMost];               // (values of its last piece - 1) * 2 + whether they are bfloat16
  int32_t count, piece;              // tensors, values of a piece

  void add(const sagnn_grad& h) {
    const int64_t pieces = ceil_div(h.n, piece);
    const void* at[2] = {h.d_in, h.d_out};
    for (int i = 0; i < (OUT ? 2 : 1); ++i) {
      low[i * kMost + count] = (uint32_t)(uintptr_t)at[i];
      high[i * kMost + count] = (uint16_t)((uintptr_t)at[i] >> 32);
    }
    end[count] = (uint16_t)((h.n - (pieces - 1) * piece - 1) * 2 + (h.dtype == SAGNN_BF16));
    first[count + 1] = first[count] + (int32_t)pieces;
    ++count;
  }
  __device__ __forceinline__ char* in(int t) const { return reinterpret_cast<char*>((uint64_t)high[t] << 32 | low[t]); }
  __device__ __forceinline__ char* out(int t) const { return in(OUT ? kMost + t : t); }
  __device__ __forceinline__ bool bf16(int t) const { return end[t] & 1; }
  // values of a piece
  __device__ __forceinline__ int values(int t, int32_t p) const { return p + 1 == first[t + 1] ? (end[t] >> 1) + 1 : piece; }
};
static_assert(kMostPiece <= 32768, "a tensor's end has 15 bits");
static_assert(sizeof(List<false>) <= kListBytes && sizeof(List<true>) <= kListBytes, "arguments of a launch");

// Tensor of a piece, by the pieces before each (64 tensors a round)
template <bool OUT>
__device__ __forceinline__ int find_tensor(const List<OUT>& l, int32_t piece) {
  const int lane = threadIdx.x & 63;
  int count = 0;
  for (int t0 = 0; t0 < l.count; t0 += 64) {
    const bool upto = t0 + lane < l.count && l.first[t0 + lane] <= piece;
    const uint64_t mask = __ballot(upto);
    count += __popcll(mask);
    if (mask != ~0ull) break;
  }
  return __builtin_amdgcn_readfirstlane(count - 1);
}

template <typename S, int V>
struct __attribute__((packed)) Packed { S x[V]; };
template <typename S, int V>
struct __attribute__((aligned(16))) Whole { S x[V]; };

// n values, 16 bytes at a time whatever their alignment
template <typename S>
__device__ __forceinline__ double sum_piece(const S* __restrict__ p, int n) {
  constexpr int V = 16 / sizeof(S);
  double s = 0.;
  int i = threadIdx.x * V;
  for (; i + 3 * kThreads * V + V <= n; i += 4 * kThreads * V) {        // (four loads in flight)
    Whole<S, V> w[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) __builtin_memcpy(&w[u], reinterpret_cast<const Packed<S, V>*>(p + i + u * kThreads * V), 16);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int e = 0; e < V; ++e) s = fma((double)(float)w[u].x[e], (double)(float)w[u].x[e], s);
  }
  for (; i + V <= n; i += kThreads * V) {
    Whole<S, V> w;
    __builtin_memcpy(&w, reinterpret_cast<const Packed<S, V>*>(p + i), 16);
#pragma unroll
    for (int e = 0; e < V; ++e) s = fma((double)(float)w.x[e], (double)(float)w.x[e], s);
  }
  for (int e = i; e < n && e < i + V; ++e) s = fma((double)(float)p[e], (double)(float)p[e], s);
  return s;
}

template <typename S>
__device__ __forceinline__ void scale_piece(const S* p, S* q, int n, float c) {
  constexpr int V = 16 / sizeof(S);
  int i = threadIdx.x * V;
  for (; i + 3 * kThreads * V + V <= n; i += 4 * kThreads * V) {
    Whole<S, V> w[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) __builtin_memcpy(&w[u], reinterpret_cast<const Packed<S, V>*>(p + i + u * kThreads * V), 16);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
#pragma unroll
      for (int e = 0; e < V; ++e) w[u].x[e] = (S)((float)w[u].x[e] * c);
      __builtin_memcpy(reinterpret_cast<Packed<S, V>*>(q + i + u * kThreads * V), &w[u], 16);
    }
  }
  for (; i + V <= n; i += kThreads * V) {
    Whole<S, V> w;
    __builtin_memcpy(&w, reinterpret_cast<const Packed<S, V>*>(p + i), 16);
#pragma unroll
    for (int e = 0; e < V; ++e) w.x[e] = (S)((float)w.x[e] * c);
    __builtin_memcpy(reinterpret_cast<Packed<S, V>*>(q + i), &w, 16);
  }
  for (int e = i; e < n && e < i + V; ++e) q[e] = (S)((float)p[e] * c);
}

__device__ __forceinline__ double block_sum(double s) {
  __shared__ double sm[kThreads / 64];
  for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = s;
  __syncthreads();
  s = sm[0];
  for (int w = 1; w < kThreads / 64; ++w) s += sm[w];
  return s;
}

__global__ __launch_bounds__(kThreads) void grad_sum_kernel(const List<false> l, double* __restrict__ sums) {
  double s = 0.;
  for (int32_t piece = blockIdx.x; piece < l.first[l.count]; piece += gridDim.x) {
    const int t = find_tensor(l, piece);
    const int32_t at = piece - l.first[t];
    const int n = l.values(t, piece);
    s += l.bf16(t) ? sum_piece(reinterpret_cast<const __bf16*>(l.in(t)) + (int64_t)at * l.piece, n)
                   : sum_piece(reinterpret_cast<const float*>(l.in(t)) + (int64_t)at * l.piece, n);
  }
  s = block_sum(s);
  if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

__device__ __forceinline__ double norm_of(const double* __restrict__ sums, int count) {
  double s = 0.;
  for (int i = threadIdx.x; i < count; i += kThreads) s += sums[i];
  return sqrt(block_sum(s));
}

__global__ __launch_bounds__(kThreads) void grad_norm_kernel(const double* __restrict__ sums, int count, float* __restrict__ norm) {
  const double n = norm_of(sums, count);
  if (threadIdx.x == 0) *norm = (float)n;
}

// Pieces in the order opposite to grad_sum_kernel's: what was read last is still in the caches.
template <bool OUT>
__global__ __launch_bounds__(kThreads) void grad_scale_kernel(const List<OUT> l, const double* __restrict__ sums, int count,
                                                              const float* __restrict__ given, double max_norm, float* __restrict__ norm) {
  const double n = given ? (double)*given : norm_of(sums, count);
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)n;
  const double ratio = max_norm / n;                 // (norm 0: infinite; NaN stays NaN)
  const float c = ratio > 1. ? 1.f : (float)ratio;
  for (int32_t piece = l.first[l.count] - 1 - (int32_t)blockIdx.x; piece >= 0; piece -= gridDim.x) {
    const int t = find_tensor(l, piece);
    if (c == 1.f && l.in(t) == l.out(t)) continue;   // (nothing changes)
    const int64_t at = (int64_t)(piece - l.first[t]) * l.piece;
    const int k = l.values(t, piece);
    if (l.bf16(t)) scale_piece(reinterpret_cast<const __bf16*>(l.in(t)) + at, reinterpret_cast<__bf16*>(l.out(t)) + at, k, c);
    else scale_piece(reinterpret_cast<const float*>(l.in(t)) + at, reinterpret_cast<float*>(l.out(t)) + at, k, c);
  }
}

int grid_of(int64_t pieces) { return (int)(pieces < kMaxBlocks ? pieces : kMaxBlocks); }

// The tensors in lists of one launch each: f(list, pieces)
template <bool OUT, typename F>
int each_list(const sagnn_grad* h, int32_t n, F f) {
  for (int32_t i = 0; i < n;) {
    List<OUT> l;
    l.count = 0;
    l.first[0] = 0;
    int64_t values = 0;
    int32_t end = i;
    int32_t tensors = 0;
    for (; end < n && tensors < List<OUT>::kMost; ++end) {
      if (h[end].n == 0) continue;
      if (tensors > 0 && values + h[end].n > (int64_t)kLeastPiece * (1 << 30)) break;
      values += h[end].n;
      ++tensors;
    }
    const int64_t each = (int64_t)round_up((size_t)ceil_div(values > 0 ? values : 1, kMaxBlocks), kLeastPiece);
    l.piece = (int32_t)(each < kMostPiece ? each : kMostPiece);
    for (; i < end; ++i) {
      if (h[i].n == 0) continue;
      l.add(h[i]);
    }
    if (!l.count) continue;
    const int rc = f(l, (int64_t)l.first[l.count]);
    if (rc != SAGNN_OK) return rc;
  }
  return SAGNN_OK;
}

struct Span { uintptr_t begin, end; bool written; };

// Types, sizes and addresses; and no two tensors share what one of them writes
int check(const sagnn_grad* h, int32_t n, bool written) {
  if (n < 0 || n > SAGNN_GRAD_MAX || (n > 0 && !h)) return SAGNN_EINVAL;
  for (int32_t i = 0; i < n; ++i) {
    const uintptr_t size = h[i].dtype == SAGNN_BF16 ? 2 : 4;
    if ((h[i].dtype != SAGNN_F32 && h[i].dtype != SAGNN_BF16) || h[i].n < 0 || h[i].n > ((int64_t)1 << 40)) return SAGNN_EINVAL;
    if (h[i].n == 0) continue;
    if ((uintptr_t)h[i].d_in >> 48 || (written && (uintptr_t)h[i].d_out >> 48)) return SAGNN_EINVAL;
    if (!h[i].d_in || ((uintptr_t)h[i].d_in & (size - 1))) return SAGNN_EINVAL;
    if (written && (!h[i].d_out || ((uintptr_t)h[i].d_out & (size - 1)))) return SAGNN_EINVAL;
  }
  if (!written) return SAGNN_OK;
  Span few[256];
  Span* s = 2 * (int64_t)n <= 256 ? few : new (std::nothrow) Span[2 * (size_t)n];
  if (!s) return SAGNN_ECAPACITY;
  size_t k = 0;
  for (int32_t i = 0; i < n; ++i) {
    if (h[i].n == 0) continue;
    const uintptr_t bytes = (uintptr_t)h[i].n * (h[i].dtype == SAGNN_BF16 ? 2 : 4), in = (uintptr_t)h[i].d_in, out = (uintptr_t)h[i].d_out;
    s[k++] = {out, out + bytes, true};
    if (in != out) s[k++] = {in, in + bytes, false};
  }
  std::sort(s, s + k, [](const Span& a, const Span& b) { return a.begin < b.begin; });
  uintptr_t any = 0, out = 0;
  bool shared = false;
  for (size_t i = 0; i < k; ++i) {
    shared |= s[i].begin < (s[i].written ? any : out);
    any = std::max(any, s[i].end);
    if (s[i].written) out = std::max(out, s[i].end);
  }
  if (s != few) delete[] s;
  return shared ? SAGNN_EINVAL : SAGNN_OK;
}

size_t ws_bytes_of(int32_t n) { return sizeof(double) * kMaxBlocks * (size_t)(ceil_div(n > 0 ? n : 1, List<false>::kMost) + 1); }

// Sums of all tensors into `sums`; how many there are
int launch_sums(const sagnn_grad* h, int32_t n, double* sums, int* count, hipStream_t s) {
  *count = 0;
  return each_list<false>(h, n, [&](const List<false>& l, int64_t pieces) {
    const int grid = grid_of(pieces);
    grad_sum_kernel<<<dim3((uint32_t)grid), kThreads, 0, s>>>(l, sums + *count);
    SAGNN_LAUNCH_CHECK();
    *count += grid;
    return (int)SAGNN_OK;
  });
}

template <bool OUT>
int launch_scale_as(const sagnn_grad* h, int32_t n, const double* sums, int count, const float* given, double max_norm, float* norm, hipStream_t s) {
  return each_list<OUT>(h, n, [&](const List<OUT>& l, int64_t pieces) {
    grad_scale_kernel<OUT><<<dim3((uint32_t)grid_of(pieces)), kThreads, 0, s>>>(l, sums, count, given, max_norm, norm);
    SAGNN_LAUNCH_CHECK();
    norm = nullptr;
    return (int)SAGNN_OK;
  });
}
int launch_scale(const sagnn_grad* h, int32_t n, const double* sums, int count, const float* given, double max_norm, float* norm, hipStream_t s) {
  bool out = false;
  for (int32_t i = 0; i < n; ++i) out |= h[i].n > 0 && h[i].d_in != h[i].d_out;
  return out ? launch_scale_as<true>(h, n, sums, count, given, max_norm, norm, s)
             : launch_scale_as<false>(h, n, sums, count, given, max_norm, norm, s);
}

}  // namespace
}  // namespace sagnn

SAGNN_EXPORT int grad_norm_workspace_bytes(int32_t n, size_t* bytes) {
  if (!bytes || n < 0 || n > SAGNN_GRAD_MAX) return SAGNN_EINVAL;
  *bytes = sagnn::ws_bytes_of(n);
  return SAGNN_OK;
}

SAGNN_EXPORT int grad_global_norm(const sagnn_grad* h_grads, int32_t n, float* d_norm, void* d_ws, size_t ws_bytes, void* stream) {
  using namespace sagnn;
  const int rc = check(h_grads, n, false);
  if (rc != SAGNN_OK) return rc;
  if (!d_norm || !d_ws || ((uintptr_t)d_norm & 3) || ((uintptr_t)d_ws & 7)) return SAGNN_EINVAL;
  if (ws_bytes < ws_bytes_of(n)) return SAGNN_ECAPACITY;
  hipStream_t s = (hipStream_t)stream;
  int count = 0;
  const int sum = launch_sums(h_grads, n, (double*)d_ws, &count, s);
  if (sum != SAGNN_OK) return sum;
  grad_norm_kernel<<<1, kThreads, 0, s>>>((const double*)d_ws, count, d_norm);
  SAGNN_LAUNCH_CHECK();
  return SAGNN_OK;
}

SAGNN_EXPORT int grad_clip_norm(const sagnn_grad* h_grads, int32_t n, double max_norm, float* d_norm, void* d_ws, size_t ws_bytes,
                                void* stream) {
  using namespace sagnn;
  if (!(max_norm > 0.) || std::isinf(max_norm)) return SAGNN_EINVAL;
  const int rc = check(h_grads, n, true);
  if (rc != SAGNN_OK) return rc;
  if (!d_norm || !d_ws || ((uintptr_t)d_norm & 3) || ((uintptr_t)d_ws & 7)) return SAGNN_EINVAL;
  if (ws_bytes < ws_bytes_of(n)) return SAGNN_ECAPACITY;
  hipStream_t s = (hipStream_t)stream;
  int count = 0;
  const int sum = launch_sums(h_grads, n, (double*)d_ws, &count, s);
  if (sum != SAGNN_OK) return sum;
  if (count == 0) {                                  // (no values: the norm is 0 and there is nothing to scale)
    grad_norm_kernel<<<1, kThreads, 0, s>>>((const double*)d_ws, 0, d_norm);
    SAGNN_LAUNCH_CHECK();
    return SAGNN_OK;
  }
  return launch_scale(h_grads, n, (const double*)d_ws, count, nullptr, max_norm, d_norm, s);
}

SAGNN_EXPORT int grad_scale_to_norm(const sagnn_grad* h_grads, int32_t n, double max_norm, const float* d_norm, void* stream) {
  using namespace sagnn;
  if (!(max_norm > 0.) || std::isinf(max_norm)) return SAGNN_EINVAL;
  const int rc = check(h_grads, n, true);
  if (rc != SAGNN_OK) return rc;
  if (!d_norm || ((uintptr_t)d_norm & 3)) return SAGNN_EINVAL;
  return launch_scale(h_grads, n, nullptr, 0, d_norm, max_norm, nullptr, (hipStream_t)stream);
}
