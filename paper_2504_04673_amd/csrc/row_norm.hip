// Operators on the rows of a matrix, one pass over them: dropout with a residual, root-mean-square norm of a residual sum (forward, into rows
// of 8 bits, backward), and the gather of rows of 8 bits.
//
// A row lies in the registers of 2 to 64 lanes of a wavefront, or of a workgroup, eight values a lane and turn: it is read once, its sum
// goes round the lanes, it is written.  Bound by those bytes.
#include <initializer_list>
#include <type_traits>
#include <utility>

#include "rows.h"

namespace sagnn {
namespace {

constexpr int kThreads = 256;

// Sum (largest) over the L lanes that share a row, L a power of two
template <typename T>
__device__ __forceinline__ T lanes_sum(T x, int L) {
  for (int d = 1; d < L; d *= 2) x += __shfl_xor(x, d);
  return x;
}
__device__ __forceinline__ float lanes_most(float x, int L) {
  for (int d = 1; d < L; d *= 2) x = fmaxf(x, __shfl_xor(x, d));
  return x;
}
// The same over a workgroup of THREADS; `place` has room for a value of every wavefront and is free again behind the call's second barrier
template <int THREADS, typename T, typename F>
__device__ __forceinline__ T team_join(T x, T* place, F join) {
  constexpr int kWaves = THREADS / 64;
  for (int d = 1; d < 64; d *= 2) x = join(x, __shfl_xor(x, d));
  if ((threadIdx.x & 63) == 0) place[threadIdx.x >> 6] = x;
  __syncthreads();
  T y = place[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) y = join(y, place[w]);
  __syncthreads();
  return y;
}

// 1 / sqrt(x) in 64 bits: the instruction's estimate, good to 2^-23 or so, and a Newton step.  Of zero and infinity the estimate is the result.
__device__ __forceinline__ float root_inverse(double x) {
  const double r = __builtin_amdgcn_rsq(x), e = __builtin_fma(-x * r, r, 1.);
  const double better = __builtin_fma(0.5 * r, e, r);
  return (float)(e == e ? better : r);
}

// x / scale, the nearest value of 32 bits.  (A product with the reciprocal is off by two units at most and sends values next to the middle between two of 8 bits to the
// other one.)  One correction by the remainder leaves a unit, a second the nearest value, as the reciprocal is (Markstein, 1990), if the remainders are whole: at 2^-10,
// below which all is zero in 8 bits, from a scale of 2^-92 on.  (2 M x 256 bfloat16 and a residual, with the gather: 826 us, with divisions 897.)
__device__ __forceinline__ float quotient(float x, float scale, float inverse, bool usual) {
  if (!usual) return scale > 0.f ? x / scale : x * 0.f;
  float q = x * inverse;
  q = __builtin_fmaf(__builtin_fmaf(-q, scale, x), inverse, q);
  return __builtin_fmaf(__builtin_fmaf(-q, scale, x), inverse, q);
}

struct RowArgs {
  const void* X; int64_t ldx;        // backward: the sums S
  const void* R; int64_t ldr;        // residual, or NULL; backward: gradient of S from elsewhere
  const void* G; int64_t ldg;        // backward: dL/dy
  int64_t m; int32_t C, eights;      // eights = ceil(C / 8)
  int32_t lanes;                     // of a row
  const float* gamma; double eps;
  Dropout drop;
  void* Y; int64_t ldy;              // y; backward: dL/dx
  void* S; int64_t lds;              // residual sum, or NULL; backward: dL/d(residual)
  float* rstd; float* scale;         // backward: rstd an input
  float* parts; float* dgamma;       // backward: rows of C sums, one a workgroup
};

// ------------------------------------------------------------------------------------------
// y = r + drop(x).  2 M x 256 bfloat16 with a residual: 507 us, 6.1 TB/s (a copy of 1 GiB: 5.1); 25 vector instructions a value, most of them the
// generator's, hide behind that.

template <typename T, bool RES>
__global__ __launch_bounds__(kThreads) void dropout_kernel(const RowArgs a) {
  const int lane = threadIdx.x & (a.lanes - 1);
  const int64_t per = kThreads / a.lanes, slot = threadIdx.x / a.lanes;
  const uint64_t offset = drop_offset(a.drop);
  for (int64_t r = blockIdx.x * per + slot; r < a.m; r += gridDim.x * per) {
    const T* x = reinterpret_cast<const T*>(a.X) + r * a.ldx;
    const T* res = reinterpret_cast<const T*>(a.R) + r * a.ldr;
    T* y = reinterpret_cast<T*>(a.Y) + r * a.ldy;
    for (int e = lane; e < a.eights; e += a.lanes) {
      const int there = a.C - e * 8;
      const auto w = load_eight(x + e * 8, there, a.C);
      TightRun<T, 8> z;
      if constexpr (RES) z = load_eight(res + e * 8, there, a.C);
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = (float)w.x[i];
      drop_eight(a.drop, offset, (uint32_t)r, (uint32_t)e, v);
      if constexpr (RES)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += (float)z.x[i];
      store_eight(y + e * 8, v, there);
    }
  }
}

// ------------------------------------------------------------------------------------------
// s = r + drop(x), y = s rstd gamma.  V turns of eight values a lane; TEAM: threads that share a row, 64: `lanes` of a wavefront.
// Squares are summed in 64 bits, so that no row of finite values overflows.  y is made of the sum before that is rounded for S.
// 1 M x 256 bfloat16 with residual and dropout 366 to 376 us, 5.5 TB/s; 2 M x 256 with a residual to 8 bits 713 to 726 us, 5.0 TB/s.  (With the next row's loads
// ahead of this row's work 531: the registers cost wavefronts.)
template <typename T, int V, int TEAM, bool EIGHT>
__global__ __launch_bounds__(TEAM == 64 ? kThreads : TEAM) void rms_norm_kernel(const RowArgs a) {
  constexpr bool kWide = TEAM > 64;
  __shared__ double room[kWide ? TEAM / 64 : 1];
  const int L = kWide ? TEAM : a.lanes, lane = kWide ? threadIdx.x : threadIdx.x & (L - 1);
  const int64_t per = kWide ? 1 : kThreads / L, slot = kWide ? 0 : threadIdx.x / L;
  const uint64_t offset = drop_offset(a.drop);
  float gamma[V][8];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int e = v * L + lane, there = a.C - e * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) gamma[v][i] = 1.f;
    if (a.gamma && there > 0) {
      const auto c = load_eight(a.gamma + e * 8, there, a.C);
#pragma unroll
      for (int i = 0; i < 8; ++i) gamma[v][i] = c.x[i];
    }
  }
  const double per_value = 1. / a.C;
  for (int64_t r = blockIdx.x * per + slot; r < a.m; r += gridDim.x * per) {      // (all lanes of a row together)
    float s[V][8];
    double squares = 0.;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int e = v * L + lane, there = a.C - e * 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) s[v][i] = 0.f;
      if (there <= 0) continue;
      const auto w = load_eight(reinterpret_cast<const T*>(a.X) + r * a.ldx + e * 8, there, a.C);
#pragma unroll
      for (int i = 0; i < 8; ++i) s[v][i] = (float)w.x[i];
      if (a.drop.cut) drop_eight(a.drop, offset, (uint32_t)r, (uint32_t)e, s[v]);
      if (a.R) {
        const auto z = load_eight(reinterpret_cast<const T*>(a.R) + r * a.ldr + e * 8, there, a.C);
#pragma unroll
        for (int i = 0; i < 8; ++i) s[v][i] += (float)z.x[i];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) squares += (double)s[v][i] * (double)s[v][i];
      if (a.S) store_eight(reinterpret_cast<T*>(a.S) + r * a.lds + e * 8, s[v], there);
    }
    if constexpr (kWide) squares = team_join<TEAM>(squares, room, [](double x, double y) { return x + y; });
    else squares = lanes_sum(squares, L);
    const float rstd = root_inverse(squares * per_value + a.eps);
    if (a.rstd && lane == 0) a.rstd[r] = rstd;
    float most = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int e = v * L + lane, there = a.C - e * 8;
      if (there <= 0) continue;
#pragma unroll
      for (int i = 0; i < 8; ++i) s[v][i] = s[v][i] * rstd * gamma[v][i];
      if constexpr (EIGHT)
#pragma unroll
        for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(s[v][i]));
      else store_eight(reinterpret_cast<T*>(a.Y) + r * a.ldy + e * 8, s[v], there);
    }
    if constexpr (EIGHT) {
      if constexpr (kWide) most = team_join<TEAM>(most, reinterpret_cast<float*>(room), [](float x, float y) { return fmaxf(x, y); });
      else most = lanes_most(most, L);
      // the largest value is 448, the type's own; a scale that is no normal number is zero, and its row
      float scale = most / 448.f;
      if (scale < 0x1p-126f) scale = 0.f;
      const float inverse = scale > 0.f ? 1.f / scale : 0.f;
      const bool usual = scale >= 0x1p-92f && scale < INFINITY;
      if (lane == 0) a.scale[r] = scale;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int e = v * L + lane, there = a.C - e * 8;
        if (there <= 0) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) s[v][i] = quotient(s[v][i], scale, inverse, usual);      // (448 and a unit at most, and that is 448 in 8 bits)
        store_bytes(reinterpret_cast<uint8_t*>(a.Y) + r * a.ldy + e * 8, to_e4m3(s[v]), there);
      }
    }
  }
}

// ------------------------------------------------------------------------------------------
// ds = rstd (g gamma - xh mean(g gamma xh)) + d with xh = s rstd; d(residual) = ds, dx = drop(ds); dgamma = sum over rows of g xh.
// A lane has the same columns of all its rows and adds up their terms for dgamma in 32 bits, kSerial of them at most; a workgroup's
// lanes are joined in 64 bits, and the workgroups by the next launch.  170 k x 602 fp32, five matrices: 426 us, 4.8 TB/s; 2 M x 100 bfloat16,
// three: 250 us, 4.8 TB/s.
constexpr int64_t kSerial = 384;

template <typename T, int V, int TEAM>
__global__ __launch_bounds__(TEAM == 64 ? kThreads : TEAM) void rms_norm_bwd_kernel(const RowArgs a) {
  constexpr bool kWide = TEAM > 64;
  __shared__ float room[kWide ? TEAM / 64 : V * 8 * kThreads];
  const int L = kWide ? TEAM : a.lanes, lane = kWide ? threadIdx.x : threadIdx.x & (L - 1);
  const int64_t per = kWide ? 1 : kThreads / L, slot = kWide ? 0 : threadIdx.x / L;
  const uint64_t offset = drop_offset(a.drop);
  float gamma[V][8];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int e = v * L + lane, there = a.C - e * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) gamma[v][i] = 1.f;
    if (a.gamma && there > 0) {
      const auto c = load_eight(a.gamma + e * 8, there, a.C);
#pragma unroll
      for (int i = 0; i < 8; ++i) gamma[v][i] = c.x[i];
    }
  }
  const float per_value = 1.f / a.C;
  float sums[V][8];
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[v][i] = 0.f;
  for (int64_t r = blockIdx.x * per + slot; r < a.m; r += gridDim.x * per) {
    float x[V][8], g[V][8], dot = 0.f;
    const float rstd = a.rstd[r];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int e = v * L + lane, there = a.C - e * 8;
      if (there <= 0) continue;
      const auto w = load_eight(reinterpret_cast<const T*>(a.X) + r * a.ldx + e * 8, there, a.C);
      const auto z = load_eight(reinterpret_cast<const T*>(a.G) + r * a.ldg + e * 8, there, a.C);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[v][i] = (float)w.x[i] * rstd;
        g[v][i] = (float)z.x[i];
        sums[v][i] += g[v][i] * x[v][i];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) g[v][i] *= gamma[v][i];
#pragma unroll
      for (int i = 0; i < 8; ++i) dot += g[v][i] * x[v][i];
    }
    if constexpr (kWide) dot = team_join<TEAM>(dot, room, [](float p, float q) { return p + q; });
    else dot = lanes_sum(dot, L);
    dot *= per_value;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int e = v * L + lane, there = a.C - e * 8;
      if (there <= 0) continue;
#pragma unroll
      for (int i = 0; i < 8; ++i) g[v][i] = rstd * (g[v][i] - x[v][i] * dot);
      if (a.R) {
        const auto d = load_eight(reinterpret_cast<const T*>(a.R) + r * a.ldr + e * 8, there, a.C);
#pragma unroll
        for (int i = 0; i < 8; ++i) g[v][i] += (float)d.x[i];
      }
      if (a.S) store_eight(reinterpret_cast<T*>(a.S) + r * a.lds + e * 8, g[v], there);
      if (a.Y) {
        if (a.drop.cut) drop_eight(a.drop, offset, (uint32_t)r, (uint32_t)e, g[v]);
        store_eight(reinterpret_cast<T*>(a.Y) + r * a.ldy + e * 8, g[v], there);
      }
    }
  }
  if (!a.dgamma) return;
  float* out = a.parts ? a.parts + (int64_t)blockIdx.x * a.C : a.dgamma;
  if constexpr (kWide) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int e = v * L + lane, there = a.C - e * 8;
      if (there > 0) store_eight(out + e * 8, sums[v], there);
    }
  } else {
    const int columns = V * L * 8;                  // of a slot
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) room[slot * columns + (v * L + lane) * 8 + i] = sums[v][i];
    __syncthreads();
    for (int c = threadIdx.x; c < a.C; c += kThreads) {
      double sum = 0.;
      for (int p = 0; p < per; ++p) sum += (double)room[p * columns + c];
      out[c] = (float)sum;
    }
  }
}

// dgamma = the workgroups' rows of sums, in 64 bits: 16 columns a workgroup, 16 threads to each
__global__ __launch_bounds__(256) void rms_norm_join_kernel(const float* __restrict__ parts, int64_t n, int32_t C, float* __restrict__ dgamma) {
  __shared__ double room[256];
  const int c = blockIdx.x * 16 + (threadIdx.x & 15);
  double sum = 0.;
  if (c < C)
#pragma unroll 8
    for (int64_t p = threadIdx.x >> 4; p < n; p += 16) sum += (double)parts[p * C + c];
  room[threadIdx.x] = sum;
  __syncthreads();
  if (threadIdx.x < 16 && c < C) {
#pragma unroll
    for (int p = 1; p < 16; ++p) sum += room[p * 16 + threadIdx.x];
    dgamma[c] = (float)sum;
  }
}

// ------------------------------------------------------------------------------------------
// out[i, :] = scale[rows[i]] q[rows[i], :]; a row out of range is zeros.  0.8 M of 2 M rows of 256 to bfloat16: 118 us, 5.2 TB/s.
template <typename T>
__global__ __launch_bounds__(kThreads) void unpack_rows_kernel(const uint8_t* __restrict__ Q, int64_t ldq, const float* __restrict__ scale, int64_t n, int32_t C,
                                                               int32_t eights, int32_t lanes, const int32_t* __restrict__ rows, int64_t N, T* __restrict__ out,
                                                               int64_t ldo) {
  const int lane = threadIdx.x & (lanes - 1);
  const int64_t per = kThreads / lanes, slot = threadIdx.x / lanes;
  for (int64_t i = blockIdx.x * per + slot; i < N; i += gridDim.x * per) {
    const int64_t r = rows ? rows[i] : i;
    const bool in = r >= 0 && r < n;
    const float s = in ? scale[r] : 0.f;
    for (int e = lane; e < eights; e += lanes) {
      const int there = C - e * 8;
      float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (in) {
        from_e4m3(load_bytes(Q + r * ldq + e * 8, there, C), v);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= s;
      }
      store_eight(out + i * ldo + e * 8, v, there);
    }
  }
}

// ------------------------------------------------------------------------------------------

int lanes_of(int32_t eights, int most) {
  int l = 2;
  while (l < eights && l < most) l *= 2;
  return l;
}
// Workgroups for m rows, `per` of them each at a time, `most` at the most
dim3 workgroups(int64_t m, int64_t per, int64_t most) {
  const int64_t n = ceil_div(m, per);
  return dim3((uint32_t)(n < most ? n : most));
}
// How many workgroups are best is measured: dropout (2 M x 256 bfloat16 and a residual) 574 us with the 2048 that the chip holds, 613 with 4096, 511 with
// one for every few rows; the norm, whose workgroups keep their scale (1 M x 256), 495 with what the chip holds, 394 with 8192, 372 with 32768, 402
// with one for every few rows; the gather (0.8 M of 2 M rows of 256) 118, 124 with 16384 and 143 with one for every few.
constexpr int64_t kDropGroups = 4000000, kNormGroups = 32768, kPackGroups = 2048;

// How a row is spread: V turns of eight values over `team` threads (64: lanes of a wavefront)
struct RowForm { int turns, team; };
RowForm row_form(int32_t eights) {
  if (eights <= 64) return {1, 64};
  if (eights <= 128) return {2, 64};
  if (eights <= 256) return {4, 64};
  if (eights <= 512) return {2, 256};
  return {2, 1024};
}
template <typename F>
int by_form(const RowForm& f, F go) {
  using std::integral_constant;
  if (f.team == 64) {
    if (f.turns == 1) return go(integral_constant<int, 1>{}, integral_constant<int, 64>{});
    if (f.turns == 2) return go(integral_constant<int, 2>{}, integral_constant<int, 64>{});
    return go(integral_constant<int, 4>{}, integral_constant<int, 64>{});
  }
  if (f.team == 256) return go(integral_constant<int, 2>{}, integral_constant<int, 256>{});
  return go(integral_constant<int, 2>{}, integral_constant<int, 1024>{});
}

// Workgroups of the backward pass: each thread has kSerial rows at most, and a workgroup enough of them that its row of sums does not count
int64_t bwd_workgroups(int64_t m, int32_t C) {
  const int32_t eights = (C + 7) / 8;
  const RowForm f = row_form(eights);
  const int64_t per = f.team == 64 ? kThreads / lanes_of(eights, 64) : 1;
  // as many as the chip holds at once (by their registers)
  const int64_t most = f.team == 64 ? (f.turns == 1 ? 6 : f.turns == 2 ? 4 : 2) * 256 : f.team == 256 ? 1024 : 256;
  int64_t n = ceil_div(m, per * 8);
  if (n > most) n = most;
  if (n < ceil_div(m, per * kSerial)) n = ceil_div(m, per * kSerial);
  return n < 1 ? 1 : n;
}
size_t bwd_bytes(int64_t m, int32_t C) {
  const int64_t n = bwd_workgroups(m, C);
  return n > 1 ? round_up((size_t)n * C * sizeof(float), 256) : 0;
}

bool valid(int32_t dtype, int64_t m, int32_t C) {
  return (dtype == SAGNN_F32 || dtype == SAGNN_BF16) && m >= 0 && m <= INT32_MAX && C >= 1 && C <= SAGNN_NORM_MAX_WIDTH;
}
uintptr_t size_of(int32_t dtype) { return dtype == SAGNN_BF16 ? 2 : 4; }
// Two outputs have nothing in common (columns beside each other are apart)
bool apart(const void* p, int64_t ldp, const void* q, int64_t ldq, int64_t m, int32_t C, uintptr_t size) {
  return !p || !q || m == 0 || (p != q && !tangled(p, ldp, q, ldq, m, C, size));
}
// An output lies in an operand's place, or apart from it
bool in_place(const void* out, int64_t ldo, const void* in, int64_t ldi, int64_t m, int32_t C, uintptr_t size) {
  return !out || !in || !tangled(out, ldo, in, ldi, m, C, size);
}
// Matrices of values of different size have no byte in common
bool disjoint(const void* p, int64_t ldp, uintptr_t size_p, const void* q, int64_t ldq, uintptr_t size_q, int64_t m, int32_t C) {
  if (!p || !q || m == 0) return true;
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return a + ((uintptr_t)(m - 1) * ldp + C) * size_p <= b || b + ((uintptr_t)(m - 1) * ldq + C) * size_q <= a;
}

}  // namespace
}  // namespace sagnn

SAGNN_EXPORT int dropout_add(int32_t dtype, const void* d_X, int64_t ldx, const void* d_R, int64_t ldr, int64_t m, int32_t C, int32_t drop, uint64_t seed,
                             uint64_t offset, const uint64_t* d_offset, int64_t row0, void* d_Y, int64_t ldy, void* stream) {
  using namespace sagnn;
  RowArgs a{};
  if (!valid(dtype, m, C) || ldx < C || ldy < C || (d_R && ldr < C) || !make_dropout(drop, seed, offset, d_offset, row0, m, &a.drop)) return SAGNN_EINVAL;
  if (m == 0) return SAGNN_OK;
  const uintptr_t size = size_of(dtype);
  if (!d_X || !d_Y || !aligned_to(d_X, size) || !aligned_to(d_R, size) || !aligned_to(d_Y, size)) return SAGNN_EINVAL;
  if (!in_place(d_Y, ldy, d_X, ldx, m, C, size) || !in_place(d_Y, ldy, d_R, ldr, m, C, size)) return SAGNN_EINVAL;
  a.X = d_X; a.ldx = ldx; a.R = d_R; a.ldr = ldr; a.m = m; a.C = C; a.eights = (C + 7) / 8; a.lanes = lanes_of(a.eights, 64); a.Y = d_Y; a.ldy = ldy;
  const dim3 grid = workgroups(m, kThreads / a.lanes, kDropGroups);
  hipStream_t s = (hipStream_t)stream;
  if (dtype == SAGNN_BF16 && d_R) dropout_kernel<__bf16, true><<<grid, kThreads, 0, s>>>(a);
  else if (dtype == SAGNN_BF16) dropout_kernel<__bf16, false><<<grid, kThreads, 0, s>>>(a);
  else if (d_R) dropout_kernel<float, true><<<grid, kThreads, 0, s>>>(a);
  else dropout_kernel<float, false><<<grid, kThreads, 0, s>>>(a);
  SAGNN_LAUNCH_CHECK();
  return SAGNN_OK;
}

SAGNN_EXPORT int rms_norm_fwd(int32_t dtype, const void* d_X, int64_t ldx, const void* d_R, int64_t ldr, int64_t m, int32_t C, const float* d_gamma,
                              double eps, int32_t drop, uint64_t seed, uint64_t offset, const uint64_t* d_offset, int64_t row0, int32_t out_type,
                              void* d_Y, int64_t ldy, float* d_scale, void* d_S, int64_t lds, float* d_rstd, void* stream) {
  using namespace sagnn;
  RowArgs a{};
  const bool eight = out_type == SAGNN_E4M3;
  if (!valid(dtype, m, C) || (!eight && out_type != dtype) || ldx < C || ldy < C || (d_R && ldr < C) || (d_S && lds < C) || !(eps >= 0.) || eps > 1e30 ||
      !make_dropout(drop, seed, offset, d_offset, row0, m, &a.drop))
    return SAGNN_EINVAL;
  if (m == 0) return SAGNN_OK;
  const uintptr_t size = size_of(dtype);
  if (!d_X || !d_Y || (eight && !d_scale) || !aligned_to(d_X, size) || !aligned_to(d_R, size) || !aligned_to(d_S, size) ||
      !aligned_to(d_Y, eight ? 1 : size) || !aligned_to(d_gamma, 4) || !aligned_to(d_scale, 4) || !aligned_to(d_rstd, 4))
    return SAGNN_EINVAL;
  if (!in_place(d_S, lds, d_X, ldx, m, C, size) || !in_place(d_S, lds, d_R, ldr, m, C, size)) return SAGNN_EINVAL;
  if (eight ? !disjoint(d_Y, ldy, 1, d_X, ldx, size, m, C) || !disjoint(d_Y, ldy, 1, d_R, ldr, size, m, C) || !disjoint(d_Y, ldy, 1, d_S, lds, size, m, C)
            : !in_place(d_Y, ldy, d_X, ldx, m, C, size) || !in_place(d_Y, ldy, d_R, ldr, m, C, size) || !apart(d_Y, ldy, d_S, lds, m, C, size))
    return SAGNN_EINVAL;
  a.X = d_X; a.ldx = ldx; a.R = d_R; a.ldr = ldr; a.m = m; a.C = C; a.eights = (C + 7) / 8; a.lanes = lanes_of(a.eights, 64); a.gamma = d_gamma; a.eps = eps;
  a.Y = d_Y; a.ldy = ldy; a.S = d_S; a.lds = lds; a.rstd = d_rstd; a.scale = d_scale;
  const RowForm f = row_form(a.eights);
  return by_form(f, [&](auto turns, auto team) {
    constexpr int V = decltype(turns)::value, TEAM = decltype(team)::value, kGroup = TEAM == 64 ? kThreads : TEAM;
    const dim3 grid = workgroups(m, TEAM == 64 ? kThreads / a.lanes : 1, kNormGroups);
    hipStream_t s = (hipStream_t)stream;
    if (dtype == SAGNN_BF16 && eight) rms_norm_kernel<__bf16, V, TEAM, true><<<grid, kGroup, 0, s>>>(a);
    else if (dtype == SAGNN_BF16) rms_norm_kernel<__bf16, V, TEAM, false><<<grid, kGroup, 0, s>>>(a);
    else if (eight) rms_norm_kernel<float, V, TEAM, true><<<grid, kGroup, 0, s>>>(a);
    else rms_norm_kernel<float, V, TEAM, false><<<grid, kGroup, 0, s>>>(a);
    SAGNN_LAUNCH_CHECK();
    return (int)SAGNN_OK;
  });
}

SAGNN_EXPORT int rms_norm_bwd_workspace_bytes(int64_t m, int32_t C, size_t* bytes) {
  using namespace sagnn;
  if (!bytes || !valid(SAGNN_F32, m, C)) return SAGNN_EINVAL;
  *bytes = bwd_bytes(m, C);
  return SAGNN_OK;
}

SAGNN_EXPORT int rms_norm_bwd(int32_t dtype, const void* d_S, int64_t lds, const void* d_G, int64_t ldg, const void* d_D, int64_t ldd, int64_t m, int32_t C,
                              const float* d_gamma, const float* d_rstd, int32_t drop, uint64_t seed, uint64_t offset, const uint64_t* d_offset,
                              int64_t row0, void* d_dX, int64_t lddx, void* d_dR, int64_t lddr, float* d_dgamma, void* d_ws, size_t ws_bytes, void* stream) {
  using namespace sagnn;
  RowArgs a{};
  if (!valid(dtype, m, C) || lds < C || ldg < C || (d_D && ldd < C) || (d_dX && lddx < C) || (d_dR && lddr < C) ||
      !make_dropout(drop, seed, offset, d_offset, row0, m, &a.drop))
    return SAGNN_EINVAL;
  const uintptr_t size = size_of(dtype);
  if ((m > 0 && (!d_S || !d_G || !d_rstd)) || !aligned_to(d_S, size) || !aligned_to(d_G, size) || !aligned_to(d_D, size) || !aligned_to(d_dX, size) ||
      !aligned_to(d_dR, size) || !aligned_to(d_gamma, 4) || !aligned_to(d_rstd, 4) || !aligned_to(d_dgamma, 4) || !aligned_to(d_ws, 4))
    return SAGNN_EINVAL;
  for (const auto& out : {std::pair<void*, int64_t>{d_dX, lddx}, std::pair<void*, int64_t>{d_dR, lddr}})
    if (!in_place(out.first, out.second, d_S, lds, m, C, size) || !in_place(out.first, out.second, d_G, ldg, m, C, size) ||
        !in_place(out.first, out.second, d_D, ldd, m, C, size))
      return SAGNN_EINVAL;
  if (!apart(d_dX, lddx, d_dR, lddr, m, C, size)) return SAGNN_EINVAL;
  const size_t need = d_dgamma ? bwd_bytes(m, C) : 0;
  if (need > 0 && !d_ws) return SAGNN_EINVAL;
  if (ws_bytes < need) return SAGNN_ECAPACITY;
  a.X = d_S; a.ldx = lds; a.R = d_D; a.ldr = ldd; a.G = d_G; a.ldg = ldg; a.m = m; a.C = C; a.eights = (C + 7) / 8; a.lanes = lanes_of(a.eights, 64);
  a.gamma = d_gamma; a.rstd = const_cast<float*>(d_rstd); a.Y = d_dX; a.ldy = lddx; a.S = d_dR; a.lds = lddr; a.dgamma = d_dgamma;
  a.parts = need ? reinterpret_cast<float*>(d_ws) : nullptr;
  const int64_t blocks = bwd_workgroups(m, C);
  hipStream_t s = (hipStream_t)stream;
  const int rc = by_form(row_form(a.eights), [&](auto turns, auto team) {        // (no rows: zeros in dgamma)
    constexpr int V = decltype(turns)::value, TEAM = decltype(team)::value, kGroup = TEAM == 64 ? kThreads : TEAM;
    if (dtype == SAGNN_BF16) rms_norm_bwd_kernel<__bf16, V, TEAM><<<dim3((uint32_t)blocks), kGroup, 0, s>>>(a);
    else rms_norm_bwd_kernel<float, V, TEAM><<<dim3((uint32_t)blocks), kGroup, 0, s>>>(a);
    SAGNN_LAUNCH_CHECK();
    return (int)SAGNN_OK;
  });
  if (rc != SAGNN_OK || !need) return rc;
  rms_norm_join_kernel<<<dim3((uint32_t)ceil_div(C, 16)), 256, 0, s>>>(a.parts, blocks, C, d_dgamma);
  SAGNN_LAUNCH_CHECK();
  return SAGNN_OK;
}

SAGNN_EXPORT int spmm_pack_rows_e4m3(const void* d_Q, int64_t ldq, const float* d_scale, int64_t n, int32_t C, const int32_t* d_rows, int64_t N,
                                     int32_t out_type, void* d_out, int64_t ldo, void* stream) {
  using namespace sagnn;
  if (!valid(out_type, 0, C) || n < 0 || n > INT32_MAX || N < 0 || N > INT32_MAX || ldq < C || ldo < C || (!d_rows && N > n)) return SAGNN_EINVAL;
  if (N == 0) return SAGNN_OK;
  const uintptr_t size = size_of(out_type);
  if (!d_out || (n > 0 && (!d_Q || !d_scale)) || !aligned_to(d_out, size) || !aligned_to(d_scale, 4) || !aligned_to(d_rows, 4)) return SAGNN_EINVAL;
  const uintptr_t q = reinterpret_cast<uintptr_t>(d_Q), o = reinterpret_cast<uintptr_t>(d_out);
  if (n > 0 && q < o + ((uintptr_t)(N - 1) * ldo + C) * size && o < q + (uintptr_t)(n - 1) * ldq + C) return SAGNN_EINVAL;
  const int32_t eights = (C + 7) / 8, lanes = lanes_of(eights, 64);
  const dim3 grid = workgroups(N, kThreads / lanes, kPackGroups);
  hipStream_t s = (hipStream_t)stream;
  const uint8_t* Q = reinterpret_cast<const uint8_t*>(d_Q);
  if (out_type == SAGNN_BF16) unpack_rows_kernel<__bf16><<<grid, kThreads, 0, s>>>(Q, ldq, d_scale, n, C, eights, lanes, d_rows, N, reinterpret_cast<__bf16*>(d_out), ldo);
  else unpack_rows_kernel<float><<<grid, kThreads, 0, s>>>(Q, ldq, d_scale, n, C, eights, lanes, d_rows, N, reinterpret_cast<float*>(d_out), ldo);
  SAGNN_LAUNCH_CHECK();
  return SAGNN_OK;
}
