// Group norm with an activation over the rows of a segment, channels last: y = act((x - mean) rstd gamma + beta), mean
// and variance over a segment's rows and a group's channels; forward and backward.
//
// Two forms.  Where the longest segment (the caller says how long) and some groups of channels fit a workgroup's registers, one
// workgroup reads them once, reduces, and writes: the bytes bound it.  Otherwise the rows are cut into chunks whatever the
// segments are, one workgroup each.  Walking along the rows, the pair (chunk c, segment b) is met at its own c + b, so that the
// sums of a segment's parts lie behind one another in a table with room for chunks + segments of them.  A launch sums
// the parts, one joins them, one writes the rows: x is read twice (dy too), the price of the dependence.
#include <type_traits>

#include "common.h"

namespace sagnn {
namespace {

constexpr int kThreads = 256;
// Terms of the gradients' sums that a thread adds up in 32 bits, one after the other: equal ones may round the same way, n/3 2^-24 of
// their sum for n
constexpr int64_t kSerial = 384;

struct NormArgs {
  const void* X; int64_t ldx;
  const void* G; int64_t ldg;        // backward: dL/dy
  void* Y; int64_t ldy;              // y, or dL/dx
  const int32_t* seg; int32_t segments; int64_t each;   // seg == NULL: `each` rows a segment
  int64_t m; int32_t C, groups, D;   // D = C / groups
  const float* gamma; const float* beta;
  float* mean; float* rstd;          // segments x groups: outputs forward, inputs backward
  double eps;
  float* dgamma; float* dbeta;
  int64_t chunk, chunks;             // rows of a chunk, chunks
  int64_t table;                     // rows of `rows`
  int64_t first;                     // forward, whole segments: segments of the launches before this one
  bool joined;                       // the workgroups that write join the parts of their segments, each for itself
  int32_t slab;                      // channels of a workgroup, where it takes whole segments
  double2* parts;                    // (chunks + segments) x groups
  float* pivots;                     // forward, segments x groups: what the sums of parts are taken from
  float2* sums;                      // backward, segments x groups: the two sums over a group, divided by its size
  // backward, table x C: sums of h xh and h, over the rows of a chunk (double2: as many are added up as it has segments) or over some
  // whole segments (float2)
  void* rows;
  template <typename Sum>
  __device__ __forceinline__ Sum* row_of(int64_t at) const { return reinterpret_cast<Sum*>(rows) + at * C; }
};

template <typename S, int V>
struct __attribute__((packed)) Packed { S x[V]; };

template <typename S, int V>
struct __attribute__((aligned(sizeof(S) * V))) Whole { S x[V]; };
template <typename S, int V>
struct Two { Whole<S, V> a, b; };

// V neighbouring values at any element's alignment
template <typename S, int V>
__device__ __forceinline__ Whole<S, V> fetch(const S* p) {
  Whole<S, V> w;
  __builtin_memcpy(&w, reinterpret_cast<const Packed<S, V>*>(p), sizeof(w));
  return w;
}
template <typename S, int V>
__device__ __forceinline__ void store(S* p, const float (&v)[V]) {
  Whole<S, V> w;
#pragma unroll
  for (int i = 0; i < V; ++i) w.x[i] = (S)v[i];
  __builtin_memcpy(reinterpret_cast<Packed<S, V>*>(p), &w, sizeof(w));
}
// (what is kept stays as it was loaded: worked out once for both uses, it took four registers a 16-byte vector more)
template <typename S, int V>
__device__ __forceinline__ void keep(Whole<S, V>& w) {
  constexpr int kBytes = sizeof(S) * V;
  if constexpr (kBytes == 4) {
    uint32_t r = __builtin_bit_cast(uint32_t, w);
    asm volatile("" : "+v"(r));
    w = __builtin_bit_cast(Whole<S, V>, r);
  } else if constexpr (kBytes > 4) {
    typedef uint32_t Raw __attribute__((ext_vector_type(kBytes / 4)));
    Raw r = __builtin_bit_cast(Raw, w);
    asm volatile("" : "+v"(r));
    w = __builtin_bit_cast(Whole<S, V>, r);
  } else {
    uint16_t r = __builtin_bit_cast(uint16_t, w);
    asm volatile("" : "+v"(r));
    w = __builtin_bit_cast(Whole<S, V>, r);
  }
}
template <typename S, int V>
__device__ __forceinline__ void store_zeros(S* p) {
  float z[V];
#pragma unroll
  for (int i = 0; i < V; ++i) z[i] = 0.f;
  store<S, V>(p, z);
}

// Rows r, r + step, ... below end: N of them are fetched before the first is used.
template <int N, typename F, typename U>
__device__ __forceinline__ void each_row(int64_t r, int64_t end, int step, F get, U use) {
  using W = decltype(get(r));
  for (; r + (N - 1) * step < end; r += N * step) {
    W w[N];
#pragma unroll
    for (int n = 0; n < N; ++n) w[n] = get(r + n * step);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int n = 0; n < N; ++n) use(r + n * step, w[n]);
  }
  for (; r < end; r += step) use(r, get(r));
}

__device__ __forceinline__ int64_t seg_row(const NormArgs& a, int64_t b) {
  if (!a.seg) return b * a.each;
  const int64_t r = a.seg[b];
  return r < 0 ? 0 : (r > a.m ? a.m : r);
}

// The segment that has `row`: the last b of 0..segments with seg[b] <= row (segments: behind them all; -1: before).
// 64 places a round.
__device__ __forceinline__ int32_t seg_find(const NormArgs& a, int64_t row) {
  if (!a.seg) return (int32_t)(row / a.each);
  const int lane = threadIdx.x & 63;
  int32_t lo = 0, n = a.segments + 1;
  while (n > 0) {
    const int32_t step = (n + 63) / 64;
    const int32_t at = lo + lane * step;
    const bool in = lane * step < n && seg_row(a, at) <= row;
    const int count = __popcll(__ballot(in));
    if (count == 0) return lo - 1;
    lo += (count - 1) * step;
    if (step == 1) return lo;
    n = n - (count - 1) * step < step ? n - (count - 1) * step : step;
  }
  return lo;
}

// Rows of a chunk segment by segment: f(segment, first row, end); segment -1 or `segments`: rows of no segment.
template <typename F>
__device__ __forceinline__ void each_part(const NormArgs& a, int64_t c, F f) {
  const int64_t r1 = (c + 1) * a.chunk < a.m ? (c + 1) * a.chunk : a.m;
  for (int64_t r = c * a.chunk; r < r1;) {
    const int32_t b = __builtin_amdgcn_readfirstlane(seg_find(a, r));
    const int64_t next = b < a.segments ? seg_row(a, b + 1) : r1;
    const int64_t end = next < r1 ? next : r1;
    if (end <= r) return;                       // (offsets that do not ascend)
    f(b, r, end);
    r = end;
  }
}

// How the threads of a workgroup lie over the channels: vectors of V, a slab of up to 256 of them at a time
struct Lay { int tx, ty, per_row, rows; };
template <int V>
__device__ __forceinline__ Lay lay(const NormArgs& a, int vec0) {
  const int vecs = a.C / V - vec0;
  Lay l;
  l.per_row = vecs < kThreads ? vecs : kThreads;
  l.rows = kThreads / l.per_row;
  l.ty = threadIdx.x / l.per_row;
  l.tx = threadIdx.x % l.per_row;
  return l;
}

// As many neighbouring lanes to each of `groups` as `threads` threads have, a power of two up to 64; and their sum
__device__ __forceinline__ int lanes_each(int groups, int threads) {
  int lanes = 64;
  while (lanes > 1 && threads / lanes < groups) lanes /= 2;
  return lanes;
}
__device__ __forceinline__ void add_lanes(double2& s, int lanes) {
  for (int d = lanes / 2; d; d /= 2) {
    s.x += __shfl_xor(s.x, d);
    s.y += __shfl_xor(s.y, d);
  }
}

// Rows of `width` pairs in LDS, one behind the other, added into the first, by halves.  All threads call it; ends with a barrier.
template <typename P>
__device__ __forceinline__ void add_rows(P* sm, int rows, int width, int threads) {
  __syncthreads();
  while (rows > 1) {
    const int half = (rows + 1) / 2;
    for (int i = threadIdx.x; i < (rows - half) * width; i += threads) {
      const P a = sm[i], b = sm[half * width + i];
      sm[i] = P{a.x + b.x, a.y + b.y};
    }
    __syncthreads();
    rows = half;
  }
}

// Sums p[], q[] per thread and channel of a slab -> per group of channels, added to acc[group].  All threads call it.
template <int V>
__device__ __forceinline__ void to_groups(const NormArgs& a, const Lay& l, int c0, const double (&p)[V], const double (&q)[V], double2* sm,
                                          double2* acc) {
  __syncthreads();
  const int width = l.per_row * V;
  if (l.ty < l.rows)
#pragma unroll
    for (int i = 0; i < V; ++i) sm[(l.ty * l.per_row + l.tx) * V + i] = make_double2(p[i], q[i]);
  add_rows(sm, l.rows, width, kThreads);
  const int g0 = c0 / a.D, g1 = (c0 + width - 1) / a.D, lanes = lanes_each(g1 - g0 + 1, kThreads);
  for (int g = g0 + threadIdx.x / lanes; g - (int)(threadIdx.x / lanes) <= g1; g += kThreads / lanes) {
    double2 s = make_double2(0., 0.);
    if (g <= g1)
      for (int c = (g * a.D < c0 ? c0 : g * a.D) + threadIdx.x % lanes; c < (g + 1) * a.D && c < c0 + width; c += lanes) {
        s.x += sm[c - c0].x;
        s.y += sm[c - c0].y;
      }
    add_lanes(s, lanes);
    if (g <= g1 && threadIdx.x % lanes == 0) {
      acc[g].x += s.x;
      acc[g].y += s.y;
    }
  }
}

// 1 / (1 + exp(-z)) by the machine's exponential and reciprocal (an ulp each; the exponent's own rounding makes |z| 2^-24 of the exponential); a
// division in its place is ten instructions.
__device__ __forceinline__ float sigmoid(float z) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504f));
}
template <int ACT>
__device__ __forceinline__ float act_value(float z) {
  if (ACT == SAGNN_ACT_RELU) return z < 0.f ? 0.f : z;
  if (ACT == SAGNN_ACT_SILU) return z * sigmoid(z);
  return z;
}
// g act'(z)
template <int ACT>
__device__ __forceinline__ float act_gradient(float g, float z) {
  if (ACT == SAGNN_ACT_RELU) return z > 0.f ? g : 0.f * g;               // (a NaN for a NaN or an infinity)
  if (ACT == SAGNN_ACT_SILU) {
    const float t = sigmoid(z);
    return g * fmaf(z * t, 1.f - t, t);
  }
  return g;
}

// What the sums over a segment and group are taken from: its first value.  Squares of what is left of the mean besides the deviation would cost
// the variance its digits: their sum is (1 + ((mean - pivot) / deviation)^2) n variances, and a value of n is at most n^(1/2) deviations
// from their mean, so that of 53 bits log2(n) are lost at worst, and two or three where the first value is no outlier.  (0 where it is
// not finite: the mean then is infinite or a NaN as the sum is.)
__device__ __forceinline__ float finite(float x) { return __builtin_isfinite(x) ? x : 0.f; }
template <typename S>
__device__ __forceinline__ float pivot_of(const NormArgs& a, int64_t row, int c) {
  return finite((float)reinterpret_cast<const S*>(a.X)[row * a.ldx + c / a.D * a.D]);
}

// Sum and sum of squares of a part, from the segment's pivots, in 64 bits
template <typename S, int V>
__global__ __launch_bounds__(kThreads) void norm_sum_kernel(const NormArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  double2* acc = reinterpret_cast<double2*>(smem);
  double2* sm = acc + a.groups;
  const S* X = reinterpret_cast<const S*>(a.X);
  const int64_t c = blockIdx.x;
  each_part(a, c, [&](int32_t b, int64_t r0, int64_t r1) {
    if (b < 0 || b >= a.segments) return;
    const int64_t lo = seg_row(a, b);
    for (int g = threadIdx.x; g < a.groups; g += kThreads) {
      acc[g] = make_double2(0., 0.);
      if (r0 == lo) a.pivots[(int64_t)b * a.groups + g] = pivot_of<S>(a, lo, g * a.D);
    }
    for (int vec0 = 0; vec0 * V < a.C; vec0 += kThreads) {
      const Lay l = lay<V>(a, vec0);
      const int ch = (vec0 + l.tx) * V;
      double p[V], q[V], from[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        p[i] = q[i] = 0.;
        from[i] = pivot_of<S>(a, lo, ch + i);
      }
      if (l.ty < l.rows)
        each_row<4>(r0 + l.ty, r1, l.rows, [&](int64_t r) { return fetch<S, V>(X + r * a.ldx + ch); }, [&](int64_t, const Whole<S, V>& w) {
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const double d = (double)(float)w.x[i] - from[i];
            p[i] += d;
            q[i] = fma(d, d, q[i]);
          }
        });
      to_groups<V>(a, l, vec0 * V, p, q, sm, acc);
    }
    __syncthreads();
    for (int g = threadIdx.x; g < a.groups; g += kThreads) a.parts[(c + b) * a.groups + g] = acc[g];
    __syncthreads();
  });
}

// Parts of a segment and group, added by `lanes` neighbouring lanes: each every lanes-th, then the lanes
__device__ __forceinline__ double2 join_parts(const NormArgs& a, int32_t b, int32_t g, int64_t lo, int64_t hi, int lanes) {
  double2 s = make_double2(0., 0.);
  if (hi > lo) {
#pragma unroll 4
    for (int64_t c = lo / a.chunk + threadIdx.x % lanes; c <= (hi - 1) / a.chunk; c += lanes) {
      const double2 p = a.parts[(c + b) * a.groups + g];
      s.x += p.x;
      s.y += p.y;
    }
  }
  add_lanes(s, lanes);
  return s;
}

// Mean and reciprocal deviation of n values by their sums from a pivot
__device__ __forceinline__ float2 moments(const NormArgs& a, double2 s, int64_t rows, double pivot) {
  const double n = rows > 0 ? (double)rows * a.D : 1.;
  const double mean = s.x / n, var = s.y / n - mean * mean;
  return make_float2((float)(pivot + mean), (float)(1. / sqrt((var < 0. ? 0. : var) + a.eps)));
}
// Backward: the two sums over the group's size
__device__ __forceinline__ float2 means(const NormArgs& a, double2 s, int64_t rows) {
  const double n = rows > 0 ? (double)rows * a.D : 1.;
  return make_float2((float)(s.x / n), (float)(s.y / n));
}

// Workgroups that join the parts of segments and groups, one for each wavefront, in turn beyond that
constexpr int64_t kMostJoins = 1 << 20;
__global__ __launch_bounds__(kThreads) void norm_join_kernel(const NormArgs a) {
  for (int64_t at = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6); at < (int64_t)a.segments * a.groups;
       at += (int64_t)gridDim.x * (kThreads / 64)) {
    const int32_t b = (int32_t)(at / a.groups), g = (int32_t)(at % a.groups);
    const int64_t lo = seg_row(a, b), hi = seg_row(a, b + 1);
    const float2 s = moments(a, join_parts(a, b, g, lo, hi, 64), hi - lo, hi > lo ? a.pivots[at] : 0.f);
    if ((threadIdx.x & 63) == 0) {
      a.mean[at] = s.x;
      a.rstd[at] = s.y;
    }
  }
}

// The same inside a workgroup that writes rows of segment b: of(sums, rows, group) of each group into `out`
template <typename F>
__device__ __forceinline__ void join_here(const NormArgs& a, int32_t b, float2* out, F of) {
  const int64_t lo = seg_row(a, b), hi = seg_row(a, b + 1);
  __syncthreads();
  const int lanes = lanes_each(a.groups, kThreads), first = threadIdx.x / lanes;
  for (int32_t g = first; g - first < a.groups; g += kThreads / lanes) {      // (all lanes stay for the sums)
    const double2 s = join_parts(a, b, g, lo, g < a.groups ? hi : lo, lanes);
    if (g < a.groups && threadIdx.x % lanes == 0) out[g] = of(s, hi - lo, g);
  }
  __syncthreads();
}

// What a vector's channels make of its values: d = x - mean, z = scale d + beta, (x - mean) rstd = rstd d.  The mean is taken off before
// anything is multiplied: values equal to it give beta, and a mean far from zero costs what its own rounding costs and no more.
// N: groups that a vector can have, 1 where a group is whole vectors, else V.
template <int V, int N>
struct Channel {
  float scale[V], beta[V], rstd[N], mean[N];
  __device__ __forceinline__ float off(float x, int i) const { return x - mean[i % N]; }
  __device__ __forceinline__ float z(float d, int i) const { return fmaf(d, scale[i], beta[i]); }
  __device__ __forceinline__ void read(const NormArgs& a, int32_t b, int ch) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int64_t g = (int64_t)b * a.groups + (ch + i) / a.D;
      rstd[i] = a.rstd[g];
      mean[i] = a.mean[g];
    }
    affine(a, ch);
  }
  // (of a vector's groups, N = V)
  __device__ __forceinline__ void read(const NormArgs& a, const float2* moments, int ch) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float2 m = moments[(ch + i) / a.D];
      mean[i] = m.x;
      rstd[i] = m.y;
    }
    affine(a, ch);
  }
  __device__ __forceinline__ void affine(const NormArgs& a, int ch) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      scale[i] = (a.gamma ? a.gamma[ch + i] : 1.f) * rstd[i % N];
      beta[i] = a.beta ? a.beta[ch + i] : 0.f;
    }
  }
};

template <typename S, int V, int ACT>
__global__ __launch_bounds__(kThreads) void norm_write_kernel(const NormArgs a) {
  const S* X = reinterpret_cast<const S*>(a.X);
  S* Y = reinterpret_cast<S*>(a.Y);
  extern __shared__ __attribute__((aligned(16))) char smem[];
  float2* here = reinterpret_cast<float2*>(smem);
  if (a.joined && blockIdx.x == 0)                          // (segments without rows are nobody's)
    for (int b = 0; b < a.segments; ++b)
      if (seg_row(a, b + 1) <= seg_row(a, b))
        for (int g = threadIdx.x; g < a.groups; g += kThreads) {
          const float2 s = moments(a, make_double2(0., 0.), 0, 0.);
          a.mean[b * a.groups + g] = s.x;
          a.rstd[b * a.groups + g] = s.y;
        }
  // (last chunk first: what was read last is still in the caches)
  each_part(a, a.chunks - 1 - blockIdx.x, [&](int32_t b, int64_t r0, int64_t r1) {
    const bool none = b < 0 || b >= a.segments;
    if (a.joined && !none) {
      join_here(a, b, here, [&](double2 s, int64_t rows, int32_t g) { return moments(a, s, rows, a.pivots[(int64_t)b * a.groups + g]); });
      if (r0 == seg_row(a, b))
        for (int g = threadIdx.x; g < a.groups; g += kThreads) {
          a.mean[b * a.groups + g] = here[g].x;
          a.rstd[b * a.groups + g] = here[g].y;
        }
    }
    for (int vec0 = 0; vec0 * V < a.C; vec0 += kThreads) {
      const Lay l = lay<V>(a, vec0);
      if (l.ty >= l.rows) continue;
      const int ch = (vec0 + l.tx) * V;
      if (none) {
        for (int64_t r = r0 + l.ty; r < r1; r += l.rows) store_zeros<S, V>(Y + r * a.ldy + ch);
        continue;
      }
      Channel<V, V> k;
      if (a.joined) k.read(a, here, ch);
      else k.read(a, b, ch);
      each_row<4>(r0 + l.ty, r1, l.rows, [&](int64_t r) { return fetch<S, V>(X + r * a.ldx + ch); }, [&](int64_t r, const Whole<S, V>& w) {
        float y[V];
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = act_value<ACT>(k.z(k.off((float)w.x[i], i), i));
        store<S, V>(Y + r * a.ldy + ch, y);
      });
    }
  });
}

template <typename S, int V, int ACT>
__global__ __launch_bounds__(kThreads) void norm_bwd_sum_kernel(const NormArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  double2* acc = reinterpret_cast<double2*>(smem);
  double2* sm = acc + a.groups;
  const S* X = reinterpret_cast<const S*>(a.X);
  const S* G = reinterpret_cast<const S*>(a.G);
  const int64_t c = blockIdx.x;
  bool first = true;
  each_part(a, c, [&](int32_t b, int64_t r0, int64_t r1) {
    if (b < 0 || b >= a.segments) return;
    for (int g = threadIdx.x; g < a.groups; g += kThreads) acc[g] = make_double2(0., 0.);
    for (int vec0 = 0; vec0 * V < a.C; vec0 += kThreads) {
      const Lay l = lay<V>(a, vec0);
      const int ch = (vec0 + l.tx) * V;
      float p[V], q[V];
      double dp[V], dq[V];
#pragma unroll
      for (int i = 0; i < V; ++i) p[i] = q[i] = 0.f;
      if (l.ty < l.rows) {
        Channel<V, V> k;
        k.read(a, b, ch);
        each_row<2>(r0 + l.ty, r1, l.rows, [&](int64_t r) { return Two<S, V>{fetch<S, V>(X + r * a.ldx + ch), fetch<S, V>(G + r * a.ldg + ch)}; },
                    [&](int64_t, const Two<S, V>& w) {
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const float d = k.off((float)w.a.x[i], i), h = act_gradient<ACT>((float)w.b.x[i], k.z(d, i));
            p[i] += h;
            q[i] = fmaf(h, d * k.rstd[i], q[i]);
          }
        });
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float gamma = a.gamma ? a.gamma[ch + i] : 1.f;
          dp[i] = (double)p[i] * gamma;
          dq[i] = (double)q[i] * gamma;
        }
      }
      to_groups<V>(a, l, vec0 * V, dp, dq, sm, acc);
      // the chunk's own sums per channel, for gamma and beta
      __syncthreads();
      float2* sf = reinterpret_cast<float2*>(sm);
      const int width = l.per_row * V;
      if (l.ty < l.rows)
#pragma unroll
        for (int i = 0; i < V; ++i) sf[(l.ty * l.per_row + l.tx) * V + i] = make_float2(q[i], p[i]);
      add_rows(sf, l.rows, width, kThreads);
      for (int x = threadIdx.x; x < width; x += kThreads) {
        double2 s = make_double2(sf[x].x, sf[x].y);
        double2* out = a.row_of<double2>(c) + vec0 * V + x;
        if (!first) {
          s.x += out->x;
          s.y += out->y;
        }
        *out = s;
      }
    }
    first = false;
    __syncthreads();
    for (int g = threadIdx.x; g < a.groups; g += kThreads) a.parts[(c + b) * a.groups + g] = acc[g];
    __syncthreads();
  });
  if (first)
    for (int x = threadIdx.x; x < a.C; x += kThreads) a.row_of<double2>(c)[x] = make_double2(0., 0.);
}

// Sixteen channels of gamma and beta: the rows of the table, THREADS / 16 at a time.  (With 64 channels for four wavefronts 1037
// rows took 67 us.)
template <int THREADS, typename Sum>
__device__ __forceinline__ void join_rows(const NormArgs& a, int32_t block) {
  __shared__ double2 sm[THREADS / 64][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int ch = block * 16 + (threadIdx.x & 15);
  double2 s = make_double2(0., 0.);
  if (ch < a.C) {
    const Sum* p = a.row_of<Sum>(0) + ch;
#pragma unroll 8
    for (int64_t c = threadIdx.x >> 4; c < a.table; c += THREADS / 16) {
      const Sum v = p[c * a.C];
      s.x += v.x;
      s.y += v.y;
    }
  }
  for (int d = 16; d < 64; d *= 2) {
    s.x += __shfl_xor(s.x, d);
    s.y += __shfl_xor(s.y, d);
  }
  if (lane < 16) sm[wave][lane] = s;
  __syncthreads();
  if (threadIdx.x < 16 && ch < a.C) {
    for (int w = 1; w < THREADS / 64; ++w) {
      s.x += sm[w][lane].x;
      s.y += sm[w][lane].y;
    }
    if (a.dgamma) a.dgamma[ch] = (float)s.x;
    if (a.dbeta) a.dbeta[ch] = (float)s.y;
  }
}

// Workgroups below `wide` join the rows of the table, the others a segment and group for each wavefront.
constexpr int kJoinThreads = 1024;
template <typename Sum>
__global__ __launch_bounds__(kJoinThreads) void norm_bwd_join_kernel(const NormArgs a, int32_t wide) {
  if ((int)blockIdx.x < wide) {
    join_rows<kJoinThreads, Sum>(a, (int32_t)blockIdx.x);
    return;
  }
  for (int64_t at = (int64_t)(blockIdx.x - wide) * (kJoinThreads / 64) + (threadIdx.x >> 6); at < (int64_t)a.segments * a.groups;
       at += (int64_t)(gridDim.x - wide) * (kJoinThreads / 64)) {
    const int32_t b = (int32_t)(at / a.groups), g = (int32_t)(at % a.groups);
    const int64_t lo = seg_row(a, b), hi = seg_row(a, b + 1);
    const float2 s = means(a, join_parts(a, b, g, lo, hi, 64), hi - lo);
    if ((threadIdx.x & 63) == 0) a.sums[at] = s;
  }
}

// dx = h gamma rstd - rstd s1 - rstd s2 xh = h scale + tilt d + level, s1 and s2 the means of the group's sums
__device__ __forceinline__ void input_line(float rstd, float2 s, float& tilt, float& level) {
  tilt = -rstd * s.y * rstd;
  level = -rstd * s.x;
}

template <typename S, int V, int ACT>
__global__ __launch_bounds__(kThreads) void norm_bwd_write_kernel(const NormArgs a) {
  const S* X = reinterpret_cast<const S*>(a.X);
  const S* G = reinterpret_cast<const S*>(a.G);
  S* Y = reinterpret_cast<S*>(a.Y);
  extern __shared__ __attribute__((aligned(16))) char smem[];
  float2* here = reinterpret_cast<float2*>(smem);
  if ((int64_t)blockIdx.x >= a.chunks) {                    // (where there is no launch between for it)
    join_rows<kThreads, double2>(a, (int32_t)(blockIdx.x - a.chunks));
    return;
  }
  each_part(a, a.chunks - 1 - blockIdx.x, [&](int32_t b, int64_t r0, int64_t r1) {
    const bool none = b < 0 || b >= a.segments;
    if (a.joined && !none) join_here(a, b, here, [&](double2 s, int64_t rows, int32_t) { return means(a, s, rows); });
    for (int vec0 = 0; vec0 * V < a.C; vec0 += kThreads) {
      const Lay l = lay<V>(a, vec0);
      if (l.ty >= l.rows) continue;
      const int ch = (vec0 + l.tx) * V;
      if (none) {
        for (int64_t r = r0 + l.ty; r < r1; r += l.rows) store_zeros<S, V>(Y + r * a.ldy + ch);
        continue;
      }
      Channel<V, V> k;
      k.read(a, b, ch);
      float tilt[V], level[V];
#pragma unroll
      for (int i = 0; i < V; ++i) input_line(k.rstd[i], a.joined ? here[(ch + i) / a.D] : a.sums[(int64_t)b * a.groups + (ch + i) / a.D], tilt[i], level[i]);
      each_row<2>(r0 + l.ty, r1, l.rows, [&](int64_t r) { return Two<S, V>{fetch<S, V>(X + r * a.ldx + ch), fetch<S, V>(G + r * a.ldg + ch)}; },
                  [&](int64_t r, const Two<S, V>& w) {
        float y[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float d = k.off((float)w.a.x[i], i), h = act_gradient<ACT>((float)w.b.x[i], k.z(d, i));
          y[i] = fmaf(h, k.scale[i], fmaf(d, tilt[i], level[i]));
        }
        store<S, V>(Y + r * a.ldy + ch, y);
      });
    }
  });
}

// ------------------------------------------------------------------------------------------
// Whole segments: a workgroup (of 64, 256 or 512 threads) has a slab of channels, whole groups and whole vectors, of one
// segment after the other.  A thread keeps up to kKept vectors in registers between the sum and the write; what a
// segment has beyond that (it is longer than the caller said) is read again.
constexpr int kMostTeam = 512, kKept = 8;
// Backward two operands are kept, as vectors of 8 bytes: half the registers for what goes with a channel.  128 registers are
// sixteen wavefronts on a CU (as vectors of 16 bytes with twice the registers, eight wavefronts: subgraphs of 250 x 256 710 us).
constexpr int kKeptBackward = 13;
constexpr int64_t kWholeLd = 1 << 16;      // (what a workgroup keeps lies within 2^31 bytes)

struct Team { int tx, ty, per_row, rows, c0, width, vec; };
template <int V>
__device__ __forceinline__ Team team(const NormArgs& a, int slab) {
  Team t;
  t.c0 = slab * a.slab;
  t.width = a.C - t.c0 < a.slab ? a.C - t.c0 : a.slab;
  t.per_row = t.width / V;
  t.rows = (int)blockDim.x / t.per_row;
  t.ty = (int)threadIdx.x / t.per_row;
  t.tx = (int)threadIdx.x % t.per_row;
  return t;
}

// Sums p[], q[] per thread and channel (N = 1: and vector) -> out[group of the slab], for all threads to read.
template <int V, int N>
__device__ __forceinline__ void team_groups(const NormArgs& a, const Team& t, const double (&p)[N], const double (&q)[N], double2* sm, double2* out) {
  const int lane = threadIdx.x & 63, waves = blockDim.x >> 6, groups = t.width / a.D;
  __syncthreads();                                          // (the last segment's sums have been read)
  if constexpr (N == 1) {                                   // a vector lies in one group
    if (t.ty < t.rows) sm[t.tx * t.rows + t.ty] = make_double2(p[0], q[0]);
    __syncthreads();
    const int each = t.rows * (a.D / V);                    // (a group's sums lie one behind the other)
    // as many lanes to a group as there are; a power of two, so that they join by shuffles
    const int lanes = lanes_each(groups, blockDim.x);
    for (int g0 = 0; g0 < groups; g0 += (int)blockDim.x / lanes) {
      const int g = g0 + (int)threadIdx.x / lanes;
      double2 v = make_double2(0., 0.);
      if (g < groups)
        for (int i = (int)threadIdx.x % lanes; i < each; i += lanes) {
          v.x += sm[g * each + i].x;
          v.y += sm[g * each + i].y;
        }
      add_lanes(v, lanes);
      if (g < groups && threadIdx.x % lanes == 0) out[g] = v;
    }
  } else {
    if (t.ty < t.rows)
#pragma unroll
      for (int i = 0; i < V; ++i) sm[t.ty * t.width + t.tx * V + i] = make_double2(p[i], q[i]);
    __syncthreads();
    for (int g = threadIdx.x >> 6; g < groups; g += waves) {
      double2 v = make_double2(0., 0.);
      for (int i = lane; i < t.rows * a.D; i += 64) {
        const double2 x = sm[i / a.D * t.width + g * a.D + i % a.D];
        v.x += x.x;
        v.y += x.y;
      }
      add_lanes(v, 64);
      if (lane == 0) out[g] = v;
    }
  }
  __syncthreads();
}

// Rows behind the last segment: zeros, by the workgroups beyond the segments'
template <typename S, int V>
__device__ __forceinline__ void team_zeros(const NormArgs& a, const Team& t, int64_t at, int64_t of) {
  const int64_t rest = seg_row(a, a.segments);
  S* Y = reinterpret_cast<S*>(a.Y) + t.c0 + t.tx * V;
  if (t.ty < t.rows)
    for (int64_t r = rest + at * t.rows + t.ty; r < a.m; r += of * t.rows) store_zeros<S, V>(Y + r * a.ldy);
}

// V values at a uniform row's address and a lane's bytes from it
template <typename S, int V>
__device__ __forceinline__ Whole<S, V> fetch_at(const void* row, uint32_t lane) {
  return fetch<S, V>(reinterpret_cast<const S*>(reinterpret_cast<const char*>(row) + lane));
}

constexpr int kBehind = 16;                // workgroups of a slab for the rows behind the last segment
// (Vectors of several groups: six wavefronts to a SIMD are worth two registers.  1 M x 100, four groups, 20000 segments: 230 us, with five 269.)
template <typename S, int V, int N, int ACT>
__global__ __launch_bounds__(kMostTeam, N > 1 ? 6 : 1) void norm_whole_kernel(const NormArgs a, int32_t slabs) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const Team t = team<V>(a, (int)(blockIdx.x % slabs));
  const int64_t b = a.first + blockIdx.x / slabs;
  if (b >= a.segments) {
    team_zeros<S, V>(a, t, b - a.segments, kBehind);
    return;
  }
  double2* sums = reinterpret_cast<double2*>(smem);
  double2* sm = sums + a.slab / a.D;
  float* pivots = reinterpret_cast<float*>(sm + blockDim.x * N);
  const int64_t lo = seg_row(a, b), hi = seg_row(a, b + 1);
  const int ch = t.c0 + t.tx * V;
  // rows lo + ty + n * t.rows: a lane's part of the address does not change
  const uint32_t vx = (uint32_t)((t.ty * a.ldx + ch) * sizeof(S)), vy = (uint32_t)((t.ty * a.ldy + ch) * sizeof(S));
  auto x_row = [&](int64_t n) { return reinterpret_cast<const S*>(a.X) + (lo + n * t.rows) * a.ldx; };
  auto y_row = [&](int64_t n) { return reinterpret_cast<char*>(reinterpret_cast<S*>(a.Y) + (lo + n * t.rows) * a.ldy); };
  const int64_t mine = t.ty < t.rows && hi - lo > t.ty ? (hi - lo - t.ty + t.rows - 1) / t.rows : 0;
  const int there = mine < kKept ? (int)mine : kKept;
  Whole<S, V> kept[kKept];
  if (hi > lo) {                                            // (what is not there is a row that is: no branches)
    const uint32_t step = (uint32_t)(t.rows * a.ldx * sizeof(S)), at = mine ? vx : (uint32_t)(ch * sizeof(S));
#pragma unroll
    for (int n = 0; n < kKept; ++n) kept[n] = fetch_at<S, V>(x_row(0), at + (n < there ? n * step : 0));
  }
  const int groups = t.width / a.D;
  for (int g = threadIdx.x; g < groups; g += blockDim.x) pivots[g] = hi > lo ? finite((float)x_row(0)[t.c0 + g * a.D]) : 0.f;
  __syncthreads();
  double p[N], q[N], from[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    p[i] = q[i] = 0.;
    from[i] = t.ty < t.rows ? pivots[(t.tx * V + i) / a.D] : 0.f;
  }
  auto add = [&](const Whole<S, V>& w) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const double d = (double)(float)w.x[i] - from[i % N];
      p[i % N] += d;
      q[i % N] = fma(d, d, q[i % N]);
    }
  };
#pragma unroll
  for (int n = 0; n < kKept; ++n) {
    keep(kept[n]);
    if (n < there) add(kept[n]);
  }
  for (int64_t n = kKept; n < mine; ++n) add(fetch_at<S, V>(x_row(n), vx));
  team_groups<V, N>(a, t, p, q, sm, sums);
  for (int g = threadIdx.x; g < groups; g += blockDim.x) {
    const float2 s = moments(a, sums[g], hi - lo, pivots[g]);
    const int64_t at = b * a.groups + t.c0 / a.D + g;
    a.mean[at] = s.x;
    a.rstd[at] = s.y;
    sums[g] = make_double2(s.x, s.y);
  }
  __syncthreads();
  if (mine == 0) return;
  Channel<V, N> k;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const double2 s = sums[(t.tx * V + i) / a.D];
    k.mean[i] = (float)s.x;
    k.rstd[i] = (float)s.y;
  }
  k.affine(a, ch);
  auto put = [&](int64_t n, const Whole<S, V>& w) {
    float y[V];
#pragma unroll
    for (int i = 0; i < V; ++i) y[i] = act_value<ACT>(k.z(k.off((float)w.x[i], i), i));
    store<S, V>(reinterpret_cast<S*>(y_row(n) + vy), y);
  };
#pragma unroll
  for (int n = 0; n < kKept; ++n) {
    keep(kept[n]);
    if (n < there) put(n, kept[n]);
  }
  for (int64_t n = kKept; n < mine; ++n) put(n, fetch_at<S, V>(x_row(n), vx));
}

// Backward: workgroups take segments in turn and keep gamma's and beta's sums until their last one.  Segments longer than the caller said,
// more than a workgroup keeps, come behind the others, in a loop of their own: beside them it would cost registers that are not
// there (a loop over further rows inside the first one: 476 us of 1 M x 256 with SiLU became 507 to 570).
template <typename S, int V, int N, int ACT>
__global__ __launch_bounds__(kMostTeam, 4) void norm_bwd_whole_kernel(const NormArgs a, int32_t slabs) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  // (a vector of several groups has their means and sums beside it)
  // g act'(z) takes g's place where that loses nothing: in fp32, and where it is g or 0
  constexpr bool kExact = sizeof(S) == 4 || ACT != SAGNN_ACT_SILU;
  constexpr int K = N == 1 ? kKeptBackward : kKeptBackward / 2;
  const Team t = team<V>(a, (int)(blockIdx.x % slabs));
  const int64_t stripe = blockIdx.x / slabs, stripes = gridDim.x / slabs;
  double2* sums = reinterpret_cast<double2*>(smem);
  double2* sm = sums + a.slab / a.D;
  float2* all = reinterpret_cast<float2*>(sm + blockDim.x * N) + threadIdx.x;     // this thread's, V of them
#pragma unroll
  for (int i = 0; i < V; ++i) all[i * blockDim.x] = make_float2(0.f, 0.f);
  const int ch = t.c0 + t.tx * V;
  const uint32_t vx = (uint32_t)((t.ty * a.ldx + ch) * sizeof(S)), vg = (uint32_t)((t.ty * a.ldg + ch) * sizeof(S)),
                 vy = (uint32_t)((t.ty * a.ldy + ch) * sizeof(S));
  auto x_row = [&](int64_t r) { return reinterpret_cast<const S*>(a.X) + r * a.ldx; };
  auto g_row = [&](int64_t r) { return reinterpret_cast<const S*>(a.G) + r * a.ldg; };
  auto y_row = [&](int64_t r) { return reinterpret_cast<char*>(reinterpret_cast<S*>(a.Y) + r * a.ldy); };
  // rows lo + ty + n * t.rows are this thread's
  auto rows_of = [&](int64_t rows) { return t.ty < t.rows && rows > t.ty ? (rows - t.ty + t.rows - 1) / t.rows : 0; };
  auto lines = [&](int64_t rows, const Channel<V, N>& k, float (&tilt)[N], float (&level)[N]) {
    const double n_values = 1. / ((double)rows * a.D);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const double2 v = sums[(t.tx * V + i) / a.D];
      input_line(k.rstd[i], make_float2((float)(v.x * n_values), (float)(v.y * n_values)), tilt[i], level[i]);
    }
  };
  auto put = [&](int64_t r, const Channel<V, N>& k, const float (&tilt)[N], const float (&level)[N], const Whole<S, V>& w, const Whole<S, V>& g, bool done) {
    float y[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float d = k.off((float)w.x[i], i), h = done ? (float)g.x[i] : act_gradient<ACT>((float)g.x[i], k.z(d, i));
      y[i] = fmaf(h, k.scale[i], fmaf(d, tilt[i % N], level[i % N]));
    }
    store<S, V>(reinterpret_cast<S*>(y_row(r) + vy), y);
  };
  bool longer = false;
  for (int64_t b = stripe; b < a.segments; b += stripes) {
    const int64_t lo = seg_row(a, b), hi = seg_row(a, b + 1);
    if (hi <= lo) continue;
    if (hi - lo > (int64_t)K * t.rows) {
      longer = true;
      continue;
    }
    const int there = (int)rows_of(hi - lo);
    Whole<S, V> x[K], h[K];
    {
      const uint32_t step_x = (uint32_t)(t.rows * a.ldx * sizeof(S)), step_g = (uint32_t)(t.rows * a.ldg * sizeof(S)),
                     at_x = there ? vx : (uint32_t)(ch * sizeof(S)), at_g = there ? vg : (uint32_t)(ch * sizeof(S));
#pragma unroll
      for (int n = 0; n < K; ++n) {
        x[n] = fetch_at<S, V>(x_row(lo), at_x + (n < there ? n * step_x : 0));
        h[n] = fetch_at<S, V>(g_row(lo), at_g + (n < there ? n * step_g : 0));
        __builtin_amdgcn_sched_barrier(0);                  // (addresses one after the other)
      }
    }
    Channel<V, N> k;
    k.read(a, (int32_t)b, ch);
    double dp[N], dq[N];
#pragma unroll
    for (int i = 0; i < N; ++i) dp[i] = dq[i] = 0.;
    {
      float p[V], q[V];
#pragma unroll
      for (int i = 0; i < V; ++i) p[i] = q[i] = 0.f;
#pragma unroll
      for (int n = 0; n < K; ++n) {
        keep(x[n]);
        keep(h[n]);
        if (n < there)
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const float d = k.off((float)x[n].x[i], i), y = act_gradient<ACT>((float)h[n].x[i], k.z(d, i));
            p[i] += y;
            q[i] = fmaf(y, d * k.rstd[i % N], q[i]);
            if (kExact) h[n].x[i] = (S)y;
          }
        __builtin_amdgcn_sched_barrier(0);                 // (one vector's temporaries at a time)
      }
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float2 s = all[i * blockDim.x];
        s.x += q[i];
        s.y += p[i];
        all[i * blockDim.x] = s;
        const float gamma = a.gamma ? a.gamma[ch + i] : 1.f;
        dp[i % N] += (double)p[i] * gamma;
        dq[i % N] += (double)q[i] * gamma;
      }
    }
    team_groups<V, N>(a, t, dp, dq, sm, sums);
    if (there == 0) continue;
    float tilt[N], level[N];
    lines(hi - lo, k, tilt, level);
#pragma unroll
    for (int n = 0; n < K; ++n) {
      keep(x[n]);
      keep(h[n]);
      if (n < there) put(lo + (int64_t)n * t.rows, k, tilt, level, x[n], h[n], kExact);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  if (longer)
#pragma unroll 1
    for (int64_t b = stripe; b < a.segments; b += stripes) {
      const int64_t lo = seg_row(a, b), hi = seg_row(a, b + 1);
      if (hi - lo <= (int64_t)K * t.rows) continue;
      const int64_t mine = rows_of(hi - lo);
      Channel<V, N> k;
      k.read(a, (int32_t)b, ch);
      double p[V], q[V], dp[N], dq[N];                     // (there may be any number of rows)
#pragma unroll
      for (int i = 0; i < V; ++i) p[i] = q[i] = 0.;
      for (int64_t n = 0; n < mine; ++n) {
        const Whole<S, V> w = fetch_at<S, V>(x_row(lo + n * t.rows), vx), g = fetch_at<S, V>(g_row(lo + n * t.rows), vg);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float d = k.off((float)w.x[i], i), y = act_gradient<ACT>((float)g.x[i], k.z(d, i));
          p[i] += y;
          q[i] = fma((double)y, (double)(d * k.rstd[i % N]), q[i]);
        }
      }
#pragma unroll
      for (int i = 0; i < N; ++i) dp[i] = dq[i] = 0.;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        all[i * blockDim.x].x += (float)q[i];
        all[i * blockDim.x].y += (float)p[i];
        const float gamma = a.gamma ? a.gamma[ch + i] : 1.f;
        dp[i % N] += p[i] * gamma;
        dq[i % N] += q[i] * gamma;
      }
      team_groups<V, N>(a, t, dp, dq, sm, sums);
      if (mine == 0) continue;
      float tilt[N], level[N];
      lines(hi - lo, k, tilt, level);
      for (int64_t n = 0; n < mine; ++n)
        put(lo + n * t.rows, k, tilt, level, fetch_at<S, V>(x_row(lo + n * t.rows), vx), fetch_at<S, V>(g_row(lo + n * t.rows), vg), false);
    }
  team_zeros<S, V>(a, t, stripe, stripes);
  // this workgroup's row of the table of gamma's and beta's sums
  __syncthreads();
  for (int rows = t.rows; rows > 1;) {                      // by halves: a thread adds what the one `half` rows below it has
    const int half = (rows + 1) / 2;
    if (t.ty + half < rows)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float2 v = all[i * blockDim.x + half * t.per_row];
        all[i * blockDim.x].x += v.x;
        all[i * blockDim.x].y += v.y;
      }
    __syncthreads();
    rows = half;
  }
  if (t.ty == 0)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float2 v = all[i * blockDim.x];
      if (stripes > 1) {
        a.row_of<float2>(stripe)[ch + i] = v;
      } else {                                              // (the only row: nothing to join)
        if (a.dgamma) a.dgamma[ch + i] = v.x;
        if (a.dbeta) a.dbeta[ch + i] = v.y;
      }
    }
}

// Values that a thread takes at a time: what 16 bytes hold, and a divisor of the width
int vector_of(int32_t dtype, int32_t C) {
  int v = dtype == SAGNN_BF16 ? 8 : 4;
  while (C % v) v /= 2;
  return v;
}

struct NormPlan { int64_t chunk, chunks; size_t parts, pivots, sums, rows, total; };
constexpr int kMostStripes = 2048;
// Segments in parts: chunks of rows, and where the sums lie
NormPlan norm_plan(int32_t dtype, int64_t m, int32_t segments, int32_t C, int32_t groups, bool backward) {
  NormPlan p{};
  // 2048 workgroups fill the chip, half of them with matrices in the caches, whose parts are joined by every workgroup; but
  // each thread has four vectors of a value or more (14530 x 8 by chunks of 2048 rows 38 us, of 512 22)
  const int64_t vectors = ceil_div(m * C, dtype == SAGNN_BF16 ? 8 : 4);
  int64_t chunks = vectors / (4 * kThreads);
  const int64_t most = vectors > (1 << 23) ? 2048 : 1024;
  chunks = chunks < 1 ? 1 : chunks > most ? most : chunks;
  p.chunk = ceil_div(m > 0 ? m : 1, chunks);
  if (backward) {
    const int64_t per_row = C / vector_of(dtype, C), serial = kSerial * (per_row < kThreads ? kThreads / per_row : 1);
    if (p.chunk > serial) p.chunk = serial;
  }
  p.chunks = ceil_div(m > 0 ? m : 1, p.chunk);
  size_t off = 0;
  auto take = [&](size_t bytes) { const size_t o = off; off += round_up(bytes, 256); return o; };
  p.parts = take((size_t)(p.chunks + segments) * groups * sizeof(double2));
  if (backward) {
    p.sums = take((size_t)segments * groups * sizeof(float2));
    p.rows = take((size_t)p.chunks * C * sizeof(double2));
  } else {
    p.pivots = take((size_t)segments * groups * sizeof(float));
  }
  p.total = off;
  return p;
}

// Whole segments: channels of a workgroup (0: not that way), workgroups beside one another, threads
struct WholePlan { int32_t slab, slabs, threads; };
WholePlan whole_plan(int64_t m, int32_t segments, int64_t max_rows, int32_t C, int32_t D, int v, int size, int kept, bool backward) {
  WholePlan w{};
  int64_t rows = max_rows > 0 && max_rows < m ? max_rows : m;
  if (rows < 1) rows = 1;
  int32_t unit = D;                                         // whole groups and whole vectors
  while (unit % v) unit += D;
  const int64_t most = (int64_t)kMostTeam * kept;          // vectors that a workgroup keeps
  int64_t units = most / (rows * (unit / v));
  if (unit / v > kMostTeam || units < 1) return w;
  if (units > kMostTeam / (unit / v)) units = kMostTeam / (unit / v);
  const int64_t all = ceil_div(C, unit);
  if (units > all) units = all;
  units = ceil_div(all, ceil_div(all, units));              // slabs of like width
  // less than a cache line of a row for each workgroup reads lines twice: where the L2s do not have them the second time
  if (units < all && units * unit * size < 128 && m * C * size > (4 << 20)) return w;
  // Few workgroups: narrower slabs where the matrix is in the L2s; and where each has still much to do, chunks share it better (three
  // segments of 415 x 896, backward: 84 workgroups 43 us, chunks 24, narrower slabs 17.5).
  const int64_t one = rows * (unit / v);
  if (segments * ceil_div(C, units * unit) < 256 && m * C * size <= (4 << 20)) {
    const int64_t narrow = one < kMostTeam ? kMostTeam / one : 1;
    if (narrow < units) units = narrow;
  }
  const int64_t vectors = one * units;
  if (segments * ceil_div(C, units * unit) < 128 && vectors > kMostTeam * (backward ? 4 : 8)) return w;
  w.slab = (int32_t)(units * unit);
  w.slabs = (int32_t)ceil_div(C, w.slab);
  w.threads = vectors <= 64 * 4 && w.slab / v <= 64 ? 64 : vectors <= 256 * 4 && w.slab / v <= 256 ? 256 : kMostTeam;
  return w;
}
// Forward: eight values only where they are of one group.  Of several, 512 threads' sums of them are 64 KB of LDS and the groups' more.
constexpr int whole_vector(int v, int D) { return v > 4 && D % v ? 4 : v; }
size_t whole_lds(const WholePlan& w, int32_t D, int v, bool backward) {
  return ((size_t)(w.slab / D) + (size_t)w.threads * (D % v == 0 ? 1 : v)) * sizeof(double2) +
         (backward ? (size_t)w.threads * v * sizeof(float2) : (size_t)(w.slab / D) * sizeof(float));
}

// How a call is carried out, and what it needs for that
struct NormForm { WholePlan whole; NormPlan parts; int64_t table; bool joined; size_t bytes; };
NormForm norm_form(int32_t dtype, int64_t m, int32_t segments, int64_t max_rows, int32_t C, int32_t groups, int64_t ld, bool backward) {
  NormForm f{};
  const int32_t D = C / groups;
  const int size = dtype == SAGNN_BF16 ? 2 : 4;
  int v = vector_of(dtype, C);
  if (backward && v * size > 8) v /= 2;
  if (!backward) v = whole_vector(v, D);
  if (m > 0 && ld <= kWholeLd) f.whole = whole_plan(m, segments, max_rows, C, D, v, size, !backward ? kKept : D % v == 0 ? kKeptBackward : kKeptBackward / 2, backward);
  if (f.whole.slab) {
    f.table = segments < kMostStripes ? segments : kMostStripes;
    if (f.table < segments / kSerial) f.table = segments / kSerial;
    if (f.table > most_blocks(f.whole.threads) / f.whole.slabs) f.table = most_blocks(f.whole.threads) / f.whole.slabs;
    f.bytes = backward && f.table > 1 ? round_up((size_t)f.table * C * sizeof(float2), 256) : 0;
  } else {
    f.parts = norm_plan(dtype, m, segments, C, groups, backward);
    f.table = m > 0 ? f.parts.chunks : 0;
    f.bytes = f.parts.total;
    // A launch less, some ten microseconds, where every workgroup can join its segments' parts: 128 KB of them at most, and few
    // segments (170003 x 100, four groups, backward 84 -> 68 us; 2 M x 256 in 32 groups would read 134 MB of sums for it).
    f.joined = m > 0 && segments <= 64 && f.parts.chunks * groups <= 8192;
  }
  return f;
}

template <typename F>
int by_act(int32_t act, F f) {
  if (act == SAGNN_ACT_RELU) return f(std::integral_constant<int, SAGNN_ACT_RELU>{});
  if (act == SAGNN_ACT_SILU) return f(std::integral_constant<int, SAGNN_ACT_SILU>{});
  return f(std::integral_constant<int, SAGNN_ACT_IDENTITY>{});
}
template <typename F>
int by_vector(int32_t dtype, int v, F f) {
  if (dtype == SAGNN_BF16) {
    if (v == 8) return f(std::integral_constant<int, 8>{}, (__bf16)0.f);
    if (v == 4) return f(std::integral_constant<int, 4>{}, (__bf16)0.f);
    if (v == 2) return f(std::integral_constant<int, 2>{}, (__bf16)0.f);
    return f(std::integral_constant<int, 1>{}, (__bf16)0.f);
  }
  if (v == 4) return f(std::integral_constant<int, 4>{}, 0.f);
  if (v == 2) return f(std::integral_constant<int, 2>{}, 0.f);
  return f(std::integral_constant<int, 1>{}, 0.f);
}

bool valid(int32_t dtype, const int32_t* d_seg, int32_t n_seg, int64_t m, int32_t C, int32_t groups, int32_t act) {
  return (dtype == SAGNN_F32 || dtype == SAGNN_BF16) && m >= 0 && m <= INT32_MAX && n_seg >= 1 && n_seg <= (1 << 26) && C >= 1 && C <= SAGNN_NORM_MAX_WIDTH && groups >= 1 &&
         groups <= SAGNN_NORM_MAX_GROUPS && C % groups == 0 && (int64_t)n_seg * groups <= INT32_MAX && act >= SAGNN_ACT_IDENTITY && act <= SAGNN_ACT_SILU &&
         (d_seg || m % n_seg == 0);
}
}  // namespace
}  // namespace sagnn

SAGNN_EXPORT int group_norm_workspace_bytes(int32_t dtype, int64_t m, int32_t n_seg, int64_t max_rows, int32_t C, int32_t n_groups,
                                            int64_t ld, int32_t backward, size_t* bytes) {
  using namespace sagnn;
  static const int32_t some = 0;
  if (!bytes || !valid(dtype, &some, n_seg, m, C, n_groups, SAGNN_ACT_IDENTITY) || max_rows < 0 || ld < C || (backward & ~1)) return SAGNN_EINVAL;
  *bytes = norm_form(dtype, m, n_seg, max_rows, C, n_groups, ld, backward != 0).bytes;
  return SAGNN_OK;
}

SAGNN_EXPORT int group_norm_act_fwd(int32_t dtype, const void* d_X, int64_t ldx, const int32_t* d_seg, int32_t n_seg, int64_t max_rows,
                                    int64_t m, int32_t C, int32_t n_groups, const float* d_gamma, const float* d_beta, double eps,
                                    int32_t act, void* d_Y, int64_t ldy, float* d_mean, float* d_rstd, void* d_ws, size_t ws_bytes,
                                    void* stream) {
  using namespace sagnn;
  if (!valid(dtype, d_seg, n_seg, m, C, n_groups, act) || max_rows < 0 || ldx < C || ldy < C || !(eps >= 0.) || eps > 1e30) return SAGNN_EINVAL;
  if (!d_mean || !d_rstd || (m > 0 && (!d_X || !d_Y))) return SAGNN_EINVAL;
  const uintptr_t size = dtype == SAGNN_BF16 ? 2 : 4;
  if (!aligned_to(d_X, size) || !aligned_to(d_Y, size) || !aligned_to(d_seg, 4) || !aligned_to(d_gamma, 4) || !aligned_to(d_beta, 4) ||
      !aligned_to(d_mean, 4) || !aligned_to(d_rstd, 4) || !aligned_to(d_ws, 16))
    return SAGNN_EINVAL;
  if (tangled(d_Y, ldy, d_X, ldx, m, C, size)) return SAGNN_EINVAL;
  const NormForm f = norm_form(dtype, m, n_seg, max_rows, C, n_groups, ldx > ldy ? ldx : ldy, false);
  const NormPlan& p = f.parts;
  const WholePlan& w = f.whole;
  if (f.bytes > 0 && !d_ws) return SAGNN_EINVAL;
  if (ws_bytes < f.bytes) return SAGNN_ECAPACITY;
  NormArgs a{};
  a.X = d_X; a.ldx = ldx; a.Y = d_Y; a.ldy = ldy; a.seg = d_seg; a.segments = n_seg; a.each = m / n_seg; a.m = m; a.C = C; a.groups = n_groups;
  a.D = C / n_groups; a.gamma = d_gamma; a.beta = d_beta; a.mean = d_mean; a.rstd = d_rstd; a.eps = eps;
  a.chunk = p.chunk; a.chunks = p.chunks; a.parts = (double2*)((char*)d_ws + p.parts); a.pivots = (float*)((char*)d_ws + p.pivots); a.slab = w.slab; a.joined = f.joined;
  hipStream_t s = (hipStream_t)stream;
  return by_act(act, [&](auto A) { return by_vector(dtype, vector_of(dtype, C), [&](auto V, auto zero) {
    constexpr int v = decltype(V)::value, ACT = decltype(A)::value;
    using S = decltype(zero);
    if (w.slab) {
      const int64_t blocks = (int64_t)n_seg + (d_seg ? kBehind : 0), most = most_blocks(w.threads) / w.slabs;
      constexpr int u = v > 4 ? 4 : v;
      const size_t lds = whole_lds(w, a.D, whole_vector(v, a.D), false);
      for (a.first = 0; a.first < blocks; a.first += most) {
        const dim3 grid((uint32_t)((blocks - a.first < most ? blocks - a.first : most) * w.slabs));
        if (a.D % v == 0) norm_whole_kernel<S, v, 1, ACT><<<grid, (uint32_t)w.threads, lds, s>>>(a, w.slabs);
        else if (a.D % u == 0) norm_whole_kernel<S, u, 1, ACT><<<grid, (uint32_t)w.threads, lds, s>>>(a, w.slabs);
        else norm_whole_kernel<S, u, u, ACT><<<grid, (uint32_t)w.threads, lds, s>>>(a, w.slabs);
        SAGNN_LAUNCH_CHECK();
      }
      return (int)SAGNN_OK;
    }
    if (m > 0) {
      norm_sum_kernel<S, v><<<dim3((uint32_t)p.chunks), kThreads, (size_t)n_groups * 16 + kThreads * v * 16, s>>>(a);
      SAGNN_LAUNCH_CHECK();
    }
    if (!a.joined) {
      const int64_t joins = ceil_div((int64_t)n_seg * n_groups, kThreads / 64);
      norm_join_kernel<<<dim3((uint32_t)(joins < kMostJoins ? joins : kMostJoins)), kThreads, 0, s>>>(a);
      SAGNN_LAUNCH_CHECK();
    }
    if (m > 0) {
      norm_write_kernel<S, v, ACT><<<dim3((uint32_t)p.chunks), kThreads, (size_t)n_groups * sizeof(float2), s>>>(a);
      SAGNN_LAUNCH_CHECK();
    }
    return (int)SAGNN_OK;
  }); });
}

SAGNN_EXPORT int group_norm_act_bwd(int32_t dtype, const void* d_X, int64_t ldx, const void* d_G, int64_t ldg, const int32_t* d_seg,
                                    int32_t n_seg, int64_t max_rows, int64_t m, int32_t C, int32_t n_groups, const float* d_gamma,
                                    const float* d_beta, int32_t act, const float* d_mean, const float* d_rstd, void* d_dX, int64_t lddx,
                                    float* d_dgamma, float* d_dbeta, void* d_ws, size_t ws_bytes, void* stream) {
  using namespace sagnn;
  if (!valid(dtype, d_seg, n_seg, m, C, n_groups, act) || max_rows < 0 || ldx < C || ldg < C || lddx < C) return SAGNN_EINVAL;
  if (!d_mean || !d_rstd || (m > 0 && (!d_X || !d_G || !d_dX))) return SAGNN_EINVAL;
  const uintptr_t size = dtype == SAGNN_BF16 ? 2 : 4;
  if (!aligned_to(d_X, size) || !aligned_to(d_G, size) || !aligned_to(d_dX, size) || !aligned_to(d_seg, 4) || !aligned_to(d_gamma, 4) ||
      !aligned_to(d_beta, 4) || !aligned_to(d_mean, 4) || !aligned_to(d_rstd, 4) || !aligned_to(d_dgamma, 4) || !aligned_to(d_dbeta, 4) ||
      !aligned_to(d_ws, 16))
    return SAGNN_EINVAL;
  if (tangled(d_dX, lddx, d_X, ldx, m, C, size) || tangled(d_dX, lddx, d_G, ldg, m, C, size)) return SAGNN_EINVAL;
  const NormForm f = norm_form(dtype, m, n_seg, max_rows, C, n_groups, ldx > ldg ? (ldx > lddx ? ldx : lddx) : (ldg > lddx ? ldg : lddx), true);
  const NormPlan& p = f.parts;
  const WholePlan& w = f.whole;
  if (!d_ws && f.bytes > 0) return SAGNN_EINVAL;
  if (ws_bytes < f.bytes) return SAGNN_ECAPACITY;
  NormArgs a{};
  a.X = d_X; a.ldx = ldx; a.G = d_G; a.ldg = ldg; a.Y = d_dX; a.ldy = lddx; a.seg = d_seg; a.segments = n_seg; a.each = m / n_seg; a.m = m;
  a.C = C; a.groups = n_groups; a.D = C / n_groups; a.gamma = d_gamma; a.beta = d_beta; a.mean = const_cast<float*>(d_mean);
  a.rstd = const_cast<float*>(d_rstd); a.dgamma = d_dgamma; a.dbeta = d_dbeta; a.chunk = p.chunk; a.chunks = p.chunks;
  a.parts = (double2*)((char*)d_ws + p.parts); a.sums = (float2*)((char*)d_ws + p.sums); a.rows = (char*)d_ws + p.rows;
  a.table = f.table; a.slab = w.slab; a.joined = f.joined;
  hipStream_t s = (hipStream_t)stream;
  return by_act(act, [&](auto A) { return by_vector(dtype, vector_of(dtype, C), [&](auto V, auto zero) {
    constexpr int v = decltype(V)::value, ACT = decltype(A)::value;
    using S = decltype(zero);
    const int32_t wide = (int32_t)ceil_div(C, 16);
    constexpr int u = v * sizeof(S) > 8 ? v / 2 : v;
    if (w.slab) {
      const size_t lds = whole_lds(w, a.D, u, true);
      const dim3 grid((uint32_t)(a.table * w.slabs));
      if (a.D % u == 0) norm_bwd_whole_kernel<S, u, 1, ACT><<<grid, (uint32_t)w.threads, lds, s>>>(a, w.slabs);
      else norm_bwd_whole_kernel<S, u, u, ACT><<<grid, (uint32_t)w.threads, lds, s>>>(a, w.slabs);
      SAGNN_LAUNCH_CHECK();
      if (a.table > 1) {
        norm_bwd_join_kernel<float2><<<dim3((uint32_t)wide), kJoinThreads, 0, s>>>(a, wide);
        SAGNN_LAUNCH_CHECK();
      }
      return (int)SAGNN_OK;
    }
    if (m > 0) {
      norm_bwd_sum_kernel<S, v, ACT><<<dim3((uint32_t)p.chunks), kThreads, (size_t)n_groups * 16 + kThreads * v * 16, s>>>(a);
      SAGNN_LAUNCH_CHECK();
    }
    if (!a.joined) {
      const int64_t joins = ceil_div((int64_t)n_seg * n_groups, kJoinThreads / 64);
      norm_bwd_join_kernel<double2><<<dim3((uint32_t)(wide + (joins < kMostJoins ? joins : kMostJoins))), kJoinThreads, 0, s>>>(a, wide);
      SAGNN_LAUNCH_CHECK();
    }
    if (m > 0) {
      norm_bwd_write_kernel<S, v, ACT><<<dim3((uint32_t)(p.chunks + (a.joined ? wide : 0))), kThreads, (size_t)n_groups * sizeof(float2), s>>>(a);
      SAGNN_LAUNCH_CHECK();
    }
    return (int)SAGNN_OK;
  }); });
}
