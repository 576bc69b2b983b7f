// Group norm with an activation over the rows of a segment, channels last: y = act((x - mean) rstd gamma + beta), mean
// and variance over a segment's rows and a group's channels; forward and backward.
//
// The rows are cut into chunks whatever the segments are, one workgroup each.  Walking along the rows, the pair (chunk
// c, segment b) is met at its own c + b, so that the sums of a segment's parts lie behind one another in a table with
// room for chunks + segments of them.  A launch sums the parts, one joins them, one writes the rows: x is read twice
// (dy too), the price of the dependence.
#include <type_traits>

#include "common.h"

namespace sagnn {
namespace {

constexpr int kThreads = 256;

struct NormArgs {
  const void* X; int64_t ldx;
  const void* G; int64_t ldg;        // backward: dL/dy
  void* Y; int64_t ldy;              // y, or dL/dx
  const int32_t* seg; int32_t segments; int64_t each;   // seg == NULL: `each` rows a segment
  int64_t m; int32_t C, groups, D;   // D = C / groups
  const float* gamma; const float* beta;
  float* mean; float* rstd;          // segments x groups: outputs forward, inputs backward
  double eps; int32_t act;
  float* dgamma; float* dbeta;
  int64_t chunk, chunks;             // rows of a chunk, chunks
  double2* parts;                    // (chunks + segments) x groups
  float2* sums;                      // backward, segments x groups: the two sums over a group, divided by its size
  float2* rows;                      // backward, chunks x C: sums of h xh and h over the rows of a chunk
};

template <typename S, int V>
struct __attribute__((packed)) Packed { S x[V]; };

// V neighbouring values at any element's alignment
template <typename S, int V>
__device__ __forceinline__ void load(const S* p, float (&v)[V]) {
  struct __attribute__((aligned(sizeof(S) * V))) Whole { S x[V]; };
  Whole w;
  __builtin_memcpy(&w, reinterpret_cast<const Packed<S, V>*>(p), sizeof(w));
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = (float)w.x[i];
}
template <typename S, int V>
__device__ __forceinline__ void store(S* p, const float (&v)[V]) {
  struct __attribute__((aligned(sizeof(S) * V))) Whole { S x[V]; };
  Whole w;
#pragma unroll
  for (int i = 0; i < V; ++i) w.x[i] = (S)v[i];
  __builtin_memcpy(reinterpret_cast<Packed<S, V>*>(p), &w, sizeof(w));
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

// Sums p[], q[] per thread and channel of a slab -> per group of channels, added to acc[group].  All threads call it.
template <int V>
__device__ __forceinline__ void to_groups(const NormArgs& a, const Lay& l, int c0, const double (&p)[V], const double (&q)[V], double2* sm,
                                          double2* acc) {
  __syncthreads();
  const int width = l.per_row * V;
  if (l.ty < l.rows)
#pragma unroll
    for (int i = 0; i < V; ++i) sm[(l.ty * l.per_row + l.tx) * V + i] = make_double2(p[i], q[i]);
  __syncthreads();
  for (int c = threadIdx.x; c < width; c += kThreads) {
    double2 s = sm[c];
    for (int y = 1; y < l.rows; ++y) {
      s.x += sm[y * width + c].x;
      s.y += sm[y * width + c].y;
    }
    sm[c] = s;
  }
  __syncthreads();
  const int g0 = c0 / a.D, g1 = (c0 + width - 1) / a.D;
  if (a.D <= 16) {
    for (int g = g0 + threadIdx.x; g <= g1; g += kThreads) {
      double2 s = acc[g];
      for (int c = g * a.D < c0 ? c0 : g * a.D; c < (g + 1) * a.D && c < c0 + width; ++c) {
        s.x += sm[c - c0].x;
        s.y += sm[c - c0].y;
      }
      acc[g] = s;
    }
  } else {
    for (int g = g0 + (threadIdx.x >> 6); g <= g1; g += kThreads / 64) {
      double2 s = make_double2(0., 0.);
      for (int c = (g * a.D < c0 ? c0 : g * a.D) + (threadIdx.x & 63); c < (g + 1) * a.D && c < c0 + width; c += 64) {
        s.x += sm[c - c0].x;
        s.y += sm[c - c0].y;
      }
      for (int d = 32; d; d >>= 1) {
        s.x += __shfl_xor(s.x, d);
        s.y += __shfl_xor(s.y, d);
      }
      if ((threadIdx.x & 63) == 0) {
        acc[g].x += s.x;
        acc[g].y += s.y;
      }
    }
  }
}

__device__ __forceinline__ float act_value(float z, int act) {
  if (act == SAGNN_ACT_RELU) return z < 0.f ? 0.f : z;
  if (act == SAGNN_ACT_SILU) return z / (1.f + __expf(-z));
  return z;
}
__device__ __forceinline__ float act_slope(float z, int act) {
  if (act == SAGNN_ACT_RELU) return z > 0.f ? 1.f : 0.f;
  if (act == SAGNN_ACT_SILU) {
    const float t = 1.f / (1.f + __expf(-z));
    return t * (1.f + z * (1.f - t));
  }
  return 1.f;
}

// Sum and sum of squares of a part, in 64 bits: whatever the mean is against the deviation, their difference holds.
template <typename S, int V>
__global__ __launch_bounds__(kThreads) void norm_sum_kernel(const NormArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  double2* acc = reinterpret_cast<double2*>(smem);
  double2* sm = acc + a.groups;
  const S* X = reinterpret_cast<const S*>(a.X);
  const int64_t c = blockIdx.x;
  each_part(a, c, [&](int32_t b, int64_t r0, int64_t r1) {
    if (b < 0 || b >= a.segments) return;
    for (int g = threadIdx.x; g < a.groups; g += kThreads) acc[g] = make_double2(0., 0.);
    for (int vec0 = 0; vec0 * V < a.C; vec0 += kThreads) {
      const Lay l = lay<V>(a, vec0);
      const int ch = (vec0 + l.tx) * V;
      double p[V], q[V];
#pragma unroll
      for (int i = 0; i < V; ++i) p[i] = q[i] = 0.;
      if (l.ty < l.rows)
        for (int64_t r = r0 + l.ty; r < r1; r += l.rows) {
          float x[V];
          load<S, V>(X + r * a.ldx + ch, x);
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const double d = x[i];
            p[i] += d;
            q[i] += d * d;
          }
        }
      to_groups<V>(a, l, vec0 * V, p, q, sm, acc);
    }
    __syncthreads();
    for (int g = threadIdx.x; g < a.groups; g += kThreads) a.parts[(c + b) * a.groups + g] = acc[g];
    __syncthreads();
  });
}

// Parts of a segment and group, added in their order (a lane every 64th, then the lanes)
__device__ __forceinline__ double2 join_parts(const NormArgs& a, int32_t b, int32_t g, int64_t lo, int64_t hi) {
  double2 s = make_double2(0., 0.);
  if (hi > lo)
    for (int64_t c = lo / a.chunk + (threadIdx.x & 63); c <= (hi - 1) / a.chunk; c += 64) {
      const double2 p = a.parts[(c + b) * a.groups + g];
      s.x += p.x;
      s.y += p.y;
    }
  for (int d = 32; d; d >>= 1) {
    s.x += __shfl_xor(s.x, d);
    s.y += __shfl_xor(s.y, d);
  }
  return s;
}

__global__ __launch_bounds__(kThreads) void norm_join_kernel(const NormArgs a) {
  const int64_t at = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  if (at >= (int64_t)a.segments * a.groups) return;
  const int32_t b = (int32_t)(at / a.groups), g = (int32_t)(at % a.groups);
  const int64_t lo = seg_row(a, b), hi = seg_row(a, b + 1);
  const double2 s = join_parts(a, b, g, lo, hi);
  if ((threadIdx.x & 63) == 0) {
    const double n = hi > lo ? (double)(hi - lo) * a.D : 1.;
    const double mean = s.x / n, var = s.y / n - mean * mean;
    a.mean[at] = (float)mean;
    a.rstd[at] = (float)(1. / sqrt((var < 0. ? 0. : var) + a.eps));
  }
}

template <typename S, int V>
__global__ __launch_bounds__(kThreads) void norm_write_kernel(const NormArgs a) {
  const S* X = reinterpret_cast<const S*>(a.X);
  S* Y = reinterpret_cast<S*>(a.Y);
  each_part(a, blockIdx.x, [&](int32_t b, int64_t r0, int64_t r1) {
    const bool none = b < 0 || b >= a.segments;
    for (int vec0 = 0; vec0 * V < a.C; vec0 += kThreads) {
      const Lay l = lay<V>(a, vec0);
      if (l.ty >= l.rows) continue;
      const int ch = (vec0 + l.tx) * V;
      float mean[V], scale[V], beta[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int64_t g = none ? 0 : (int64_t)b * a.groups + (ch + i) / a.D;
        mean[i] = none ? 0.f : a.mean[g];
        scale[i] = (none ? 0.f : a.rstd[g]) * (a.gamma ? a.gamma[ch + i] : 1.f);
        beta[i] = a.beta ? a.beta[ch + i] : 0.f;
      }
      for (int64_t r = r0 + l.ty; r < r1; r += l.rows) {
        float x[V];
        load<S, V>(X + r * a.ldx + ch, x);
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = none ? 0.f : act_value((x[i] - mean[i]) * scale[i] + beta[i], a.act);
        store<S, V>(Y + r * a.ldy + ch, x);
      }
    }
  });
}

// What a channel's values need backward
template <int V>
struct Channel {
  float mean[V], rstd[V], gamma[V], beta[V];
  __device__ __forceinline__ void read(const NormArgs& a, int32_t b, int ch) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t g = (int64_t)b * a.groups + (ch + i) / a.D;
      mean[i] = a.mean[g];
      rstd[i] = a.rstd[g];
      gamma[i] = a.gamma ? a.gamma[ch + i] : 1.f;
      beta[i] = a.beta ? a.beta[ch + i] : 0.f;
    }
  }
};

template <typename S, int V>
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
        Channel<V> k;
        k.read(a, b, ch);
        for (int64_t r = r0 + l.ty; r < r1; r += l.rows) {
          float x[V], h[V];
          load<S, V>(X + r * a.ldx + ch, x);
          load<S, V>(G + r * a.ldg + ch, h);
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const float xh = (x[i] - k.mean[i]) * k.rstd[i];
            h[i] *= act_slope(xh * k.gamma[i] + k.beta[i], a.act);
            p[i] += h[i];
            q[i] += h[i] * xh;
          }
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
          dp[i] = (double)p[i] * k.gamma[i];
          dq[i] = (double)q[i] * k.gamma[i];
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
      __syncthreads();
      for (int x = threadIdx.x; x < width; x += kThreads) {
        float2 s = sf[x];
        for (int y = 1; y < l.rows; ++y) {
          s.x += sf[y * width + x].x;
          s.y += sf[y * width + x].y;
        }
        float2* out = a.rows + c * a.C + vec0 * V + x;
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
    for (int x = threadIdx.x; x < a.C; x += kThreads) a.rows[c * a.C + x] = make_float2(0.f, 0.f);
}

// Workgroups below `wide`: 64 channels of gamma and beta each, a row of the table for each wavefront in turn; the others:
// a segment and group for each wavefront.
__global__ __launch_bounds__(kThreads) void norm_bwd_join_kernel(const NormArgs a, int32_t wide) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if ((int)blockIdx.x < wide) {
    __shared__ double2 sm[kThreads];
    const int ch = (int)blockIdx.x * 64 + lane;
    double2 s = make_double2(0., 0.);
    if (ch < a.C)
      for (int64_t c = wave; c < a.chunks; c += kThreads / 64) {
        const float2 p = a.rows[c * a.C + ch];
        s.x += p.x;
        s.y += p.y;
      }
    sm[threadIdx.x] = s;
    __syncthreads();
    if (wave == 0 && ch < a.C) {
      for (int w = 1; w < kThreads / 64; ++w) {
        s.x += sm[w * 64 + lane].x;
        s.y += sm[w * 64 + lane].y;
      }
      if (a.dgamma) a.dgamma[ch] = (float)s.x;
      if (a.dbeta) a.dbeta[ch] = (float)s.y;
    }
    return;
  }
  const int64_t at = (int64_t)(blockIdx.x - wide) * (kThreads / 64) + wave;
  if (at >= (int64_t)a.segments * a.groups) return;
  const int32_t b = (int32_t)(at / a.groups), g = (int32_t)(at % a.groups);
  const int64_t lo = seg_row(a, b), hi = seg_row(a, b + 1);
  const double2 s = join_parts(a, b, g, lo, hi);
  const double n = hi > lo ? (double)(hi - lo) * a.D : 1.;
  if (lane == 0) a.sums[at] = make_float2((float)(s.x / n), (float)(s.y / n));
}

template <typename S, int V>
__global__ __launch_bounds__(kThreads) void norm_bwd_write_kernel(const NormArgs a) {
  const S* X = reinterpret_cast<const S*>(a.X);
  const S* G = reinterpret_cast<const S*>(a.G);
  S* Y = reinterpret_cast<S*>(a.Y);
  each_part(a, blockIdx.x, [&](int32_t b, int64_t r0, int64_t r1) {
    const bool none = b < 0 || b >= a.segments;
    for (int vec0 = 0; vec0 * V < a.C; vec0 += kThreads) {
      const Lay l = lay<V>(a, vec0);
      if (l.ty >= l.rows) continue;
      const int ch = (vec0 + l.tx) * V;
      Channel<V> k;
      float2 s[V];
      if (!none) {
        k.read(a, b, ch);
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = a.sums[(int64_t)b * a.groups + (ch + i) / a.D];
      }
      for (int64_t r = r0 + l.ty; r < r1; r += l.rows) {
        float x[V], h[V];
        if (none) {
#pragma unroll
          for (int i = 0; i < V; ++i) x[i] = 0.f;
        } else {
          load<S, V>(X + r * a.ldx + ch, x);
          load<S, V>(G + r * a.ldg + ch, h);
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const float xh = (x[i] - k.mean[i]) * k.rstd[i];
            h[i] *= act_slope(xh * k.gamma[i] + k.beta[i], a.act);
            x[i] = (h[i] * k.gamma[i] - s[i].x - xh * s[i].y) * k.rstd[i];
          }
        }
        store<S, V>(Y + r * a.ldy + ch, x);
      }
    }
  });
}

// Values that a thread takes at a time: what 16 bytes hold, and a divisor of the width
int vector_of(int32_t dtype, int32_t C) {
  int v = dtype == SAGNN_BF16 ? 8 : 4;
  while (C % v) v /= 2;
  return v;
}

struct NormPlan { int64_t chunk, chunks; size_t parts, sums, rows, total; };
NormPlan norm_plan(int64_t m, int32_t segments, int32_t C, int32_t groups) {
  NormPlan p{};
  // 2048 workgroups fill the chip; a chunk has eight rows of 256 threads or more
  int64_t least = ceil_div(8 * 2048, C);
  if (least < 8) least = 8;
  p.chunk = ceil_div(m > 0 ? m : 1, 2048);
  if (p.chunk < least) p.chunk = least;
  p.chunks = ceil_div(m > 0 ? m : 1, p.chunk);
  size_t off = 0;
  auto take = [&](size_t bytes) { const size_t o = off; off += round_up(bytes, 256); return o; };
  p.parts = take((size_t)(p.chunks + segments) * groups * sizeof(double2));
  p.sums = take((size_t)segments * groups * sizeof(float2));
  p.rows = take((size_t)p.chunks * C * sizeof(float2));
  p.total = off;
  return p;
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
bool aligned_to(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

}  // namespace
}  // namespace sagnn

SAGNN_EXPORT int group_norm_workspace_bytes(int64_t m, int32_t n_seg, int32_t C, int32_t n_groups, size_t* bytes) {
  using namespace sagnn;
  static const int32_t some = 0;
  if (!bytes || !valid(SAGNN_F32, &some, n_seg, m, C, n_groups, SAGNN_ACT_IDENTITY)) return SAGNN_EINVAL;
  *bytes = norm_plan(m, n_seg, C, n_groups).total;
  return SAGNN_OK;
}

SAGNN_EXPORT int group_norm_act_fwd(int32_t dtype, const void* d_X, int64_t ldx, const int32_t* d_seg, int32_t n_seg, int64_t max_rows,
                                    int64_t m, int32_t C, int32_t n_groups, const float* d_gamma, const float* d_beta, double eps,
                                    int32_t act, void* d_Y, int64_t ldy, float* d_mean, float* d_rstd, void* d_ws, size_t ws_bytes,
                                    void* stream) {
  using namespace sagnn;
  if (!valid(dtype, d_seg, n_seg, m, C, n_groups, act) || max_rows < 0 || ldx < C || ldy < C || !(eps >= 0.) || eps > 1e30) return SAGNN_EINVAL;
  if (!d_mean || !d_rstd || !d_ws || (m > 0 && (!d_X || !d_Y))) return SAGNN_EINVAL;
  const uintptr_t size = dtype == SAGNN_BF16 ? 2 : 4;
  if (!aligned_to(d_X, size) || !aligned_to(d_Y, size) || !aligned_to(d_seg, 4) || !aligned_to(d_gamma, 4) || !aligned_to(d_beta, 4) ||
      !aligned_to(d_mean, 4) || !aligned_to(d_rstd, 4) || !aligned_to(d_ws, 16))
    return SAGNN_EINVAL;
  const NormPlan p = norm_plan(m, n_seg, C, n_groups);
  if (ws_bytes < p.total) return SAGNN_ECAPACITY;
  NormArgs a{};
  a.X = d_X; a.ldx = ldx; a.Y = d_Y; a.ldy = ldy; a.seg = d_seg; a.segments = n_seg; a.each = m / n_seg; a.m = m; a.C = C; a.groups = n_groups;
  a.D = C / n_groups; a.gamma = d_gamma; a.beta = d_beta; a.mean = d_mean; a.rstd = d_rstd; a.eps = eps; a.act = act;
  a.chunk = p.chunk; a.chunks = p.chunks; a.parts = (double2*)((char*)d_ws + p.parts);
  hipStream_t s = (hipStream_t)stream;
  return by_vector(dtype, vector_of(dtype, C), [&](auto V, auto zero) {
    constexpr int v = decltype(V)::value;
    using S = decltype(zero);
    if (m > 0) {
      norm_sum_kernel<S, v><<<dim3((uint32_t)p.chunks), kThreads, (size_t)n_groups * 16 + kThreads * v * 16, s>>>(a);
      SAGNN_LAUNCH_CHECK();
    }
    norm_join_kernel<<<dim3((uint32_t)ceil_div((int64_t)n_seg * n_groups, kThreads / 64)), kThreads, 0, s>>>(a);
    SAGNN_LAUNCH_CHECK();
    if (m > 0) {
      norm_write_kernel<S, v><<<dim3((uint32_t)p.chunks), kThreads, 0, s>>>(a);
      SAGNN_LAUNCH_CHECK();
    }
    return (int)SAGNN_OK;
  });
}

SAGNN_EXPORT int group_norm_act_bwd(int32_t dtype, const void* d_X, int64_t ldx, const void* d_G, int64_t ldg, const int32_t* d_seg,
                                    int32_t n_seg, int64_t max_rows, int64_t m, int32_t C, int32_t n_groups, const float* d_gamma,
                                    const float* d_beta, int32_t act, const float* d_mean, const float* d_rstd, void* d_dX, int64_t lddx,
                                    float* d_dgamma, float* d_dbeta, void* d_ws, size_t ws_bytes, void* stream) {
  using namespace sagnn;
  if (!valid(dtype, d_seg, n_seg, m, C, n_groups, act) || max_rows < 0 || ldx < C || ldg < C || lddx < C) return SAGNN_EINVAL;
  if (!d_mean || !d_rstd || !d_ws || (m > 0 && (!d_X || !d_G || !d_dX))) return SAGNN_EINVAL;
  const uintptr_t size = dtype == SAGNN_BF16 ? 2 : 4;
  if (!aligned_to(d_X, size) || !aligned_to(d_G, size) || !aligned_to(d_dX, size) || !aligned_to(d_seg, 4) || !aligned_to(d_gamma, 4) ||
      !aligned_to(d_beta, 4) || !aligned_to(d_mean, 4) || !aligned_to(d_rstd, 4) || !aligned_to(d_dgamma, 4) || !aligned_to(d_dbeta, 4) ||
      !aligned_to(d_ws, 16))
    return SAGNN_EINVAL;
  const NormPlan p = norm_plan(m, n_seg, C, n_groups);
  if (ws_bytes < p.total) return SAGNN_ECAPACITY;
  NormArgs a{};
  a.X = d_X; a.ldx = ldx; a.G = d_G; a.ldg = ldg; a.Y = d_dX; a.ldy = lddx; a.seg = d_seg; a.segments = n_seg; a.each = m / n_seg; a.m = m;
  a.C = C; a.groups = n_groups; a.D = C / n_groups; a.gamma = d_gamma; a.beta = d_beta; a.mean = const_cast<float*>(d_mean);
  a.rstd = const_cast<float*>(d_rstd); a.act = act; a.dgamma = d_dgamma; a.dbeta = d_dbeta; a.chunk = p.chunk; a.chunks = p.chunks;
  a.parts = (double2*)((char*)d_ws + p.parts); a.sums = (float2*)((char*)d_ws + p.sums); a.rows = (float2*)((char*)d_ws + p.rows);
  if (m == 0) a.chunks = 0;
  hipStream_t s = (hipStream_t)stream;
  return by_vector(dtype, vector_of(dtype, C), [&](auto V, auto zero) {
    constexpr int v = decltype(V)::value;
    using S = decltype(zero);
    if (m > 0) {
      norm_bwd_sum_kernel<S, v><<<dim3((uint32_t)p.chunks), kThreads, (size_t)n_groups * 16 + kThreads * v * 16, s>>>(a);
      SAGNN_LAUNCH_CHECK();
    }
    const int32_t wide = (int32_t)ceil_div(C, 64);
    norm_bwd_join_kernel<<<dim3((uint32_t)(wide + ceil_div((int64_t)n_seg * n_groups, kThreads / 64))), kThreads, 0, s>>>(a, wide);
    SAGNN_LAUNCH_CHECK();
    if (m > 0) {
      norm_bwd_write_kernel<S, v><<<dim3((uint32_t)p.chunks), kThreads, 0, s>>>(a);
      SAGNN_LAUNCH_CHECK();
    }
    return (int)SAGNN_OK;
  });
}
