// Rows of a matrix eight values a lane: loads and stores at any element's alignment, and the generator of dropout's mask.
#pragma once
#include "common.h"

namespace sagnn {

template <typename S, int N>
struct __attribute__((packed)) LooseRun { S x[N]; };
template <typename S, int N>
struct __attribute__((aligned(sizeof(S) * N))) TightRun { S x[N]; };

// Elements of 2 or 4 bytes in words, moved down by n (0 to 7) where `tail`: zeros come in behind
template <int BYTES, int N>
__device__ __forceinline__ void move_down(uint32_t (&w)[N], int n, bool tail) {
  constexpr int kPer = 4 / BYTES;
#pragma unroll
  for (int bit = 4; bit >= kPer; bit /= 2)
    if (n & bit)                                  // (the same for every row)
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = tail ? (i + bit / kPer < N ? w[i + bit / kPer] : 0u) : w[i];
  if (BYTES == 2 && (n & 1))
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = tail ? w[i] >> 16 | (i + 1 < N ? w[i + 1] << 16 : 0u) : w[i];
}
// Values 8 e to 8 e + 8 of a row of `width`, p being the first and `there` (1 and more) up to the row's end; zeros behind it.  The last values of a row
// that is no whole eights are loaded with what is before them and moved into place, so that all lanes load at once.  (In a branch of their own
// they wait for the others' loads: gradients of 2 M x 100 bfloat16 477 us that way, 327 this way.)
template <typename S>
__device__ __forceinline__ TightRun<S, 8> load_eight(const S* p, int there, int width) {
  TightRun<S, 8> w;
  if (width >= 8) {
    const bool tail = there < 8;
    uint32_t v[sizeof(w) / 4];
    __builtin_memcpy(v, reinterpret_cast<const LooseRun<S, 8>*>(p + (tail ? there - 8 : 0)), sizeof(w));
    move_down<sizeof(S)>(v, -width & 7, tail);
    __builtin_memcpy(&w, v, sizeof(w));
    return w;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) w.x[i] = i < there ? p[i] : (S)0.f;
  return w;
}
template <typename S>
__device__ __forceinline__ void store_eight(S* p, const float (&y)[8], int there) {
  TightRun<S, 8> w;
#pragma unroll
  for (int i = 0; i < 8; ++i) w.x[i] = (S)y[i];
  if (there >= 8) {
    __builtin_memcpy(reinterpret_cast<LooseRun<S, 8>*>(p), &w, sizeof(w));
    return;
  }
  if (there >= 4) __builtin_memcpy(reinterpret_cast<LooseRun<S, 4>*>(p), &w, sizeof(w) / 2);
#pragma unroll
  for (int i = 0; i < 7; ++i)
    if (i < there && i >= (there & 4)) p[i] = w.x[i];
}

// Eight values of e4m3 (OCP: largest 448), to nearest even; none may be as much as 464, the middle to what would be next.  Two at a time into a half of a word.
__device__ __forceinline__ uint2 to_e4m3(const float (&v)[8]) {
  int lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false), hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4], v[5], 0, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6], v[7], hi, true);
  return make_uint2((uint32_t)lo, (uint32_t)hi);
}
__device__ __forceinline__ void from_e4m3(uint2 w, float (&v)[8]) {
  typedef float two __attribute__((ext_vector_type(2)));
  const two a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.x, true);
  const two c = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.y, false), d = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.y, true);
  v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y; v[4] = c.x; v[5] = c.y; v[6] = d.x; v[7] = d.y;
}
__device__ __forceinline__ void store_bytes(uint8_t* p, uint2 w, int there) {
  if (there >= 8) {
    __builtin_memcpy(reinterpret_cast<LooseRun<uint8_t, 8>*>(p), &w, 8);
    return;
  }
#pragma unroll
  for (int i = 0; i < 7; ++i)
    if (i < there) p[i] = (uint8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
}
__device__ __forceinline__ uint2 load_bytes(const uint8_t* p, int there, int width) {
  uint64_t w = 0;
  if (width >= 8) {
    const bool tail = there < 8;
    __builtin_memcpy(&w, reinterpret_cast<const LooseRun<uint8_t, 8>*>(p + (tail ? there - 8 : 0)), 8);
    w >>= tail ? (-width & 7) * 8 : 0;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < there) w |= (uint64_t)p[i] << (8 * i);
  }
  return make_uint2((uint32_t)w, (uint32_t)(w >> 32));
}

// Dropout's mask is no memory but a function: ten rounds of Philox-4x32 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy
// as 1, 2, 3", 2011) over (column / 8, row, offset) under the seed give 128 bits, 16 for each of eight columns.  Those below `cut` 65536ths fall.
// Sixteen bits a value: 20 products of 32 bits serve eight values, so that traffic stays the bound; a probability is good to 2^-17.
struct Dropout {
  uint32_t cut;                    // 0: none
  float scale;                     // of what is kept: 65536 / (65536 - cut)
  uint32_t seed0, seed1;
  uint64_t offset;
  const uint64_t* d_offset;        // added to it where there is one
  uint32_t row0;                   // number of the first row
};
inline bool make_dropout(int32_t drop, uint64_t seed, uint64_t offset, const uint64_t* d_offset, int64_t row0, int64_t m, Dropout* d) {
  if (drop < 0 || drop > 65536 || row0 < 0 || row0 > (int64_t(1) << 32) - m || !aligned_to(d_offset, 8)) return false;
  *d = Dropout{(uint32_t)drop, drop < 65536 ? (float)(65536.0 / (65536 - drop)) : 0.f, (uint32_t)seed, (uint32_t)(seed >> 32), offset, d_offset, (uint32_t)row0};
  return true;
}
__device__ __forceinline__ uint64_t drop_offset(const Dropout& d) { return d.offset + (d.d_offset ? *d.d_offset : 0); }

__device__ __forceinline__ uint4 philox(uint4 c, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = (uint64_t)c.x * 0xD2511F53u, b = (uint64_t)c.z * 0xCD9E8D57u;
    c = make_uint4((uint32_t)(b >> 32) ^ c.y ^ k0, (uint32_t)b, (uint32_t)(a >> 32) ^ c.w ^ k1, (uint32_t)a);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return c;
}
// Eight values of row `row` (counted from the call's first), columns 8 `eight` on
__device__ __forceinline__ void drop_eight(const Dropout& d, uint64_t offset, uint32_t row, uint32_t eight, float (&v)[8]) {
  const uint4 r = philox(make_uint4(eight, d.row0 + row, (uint32_t)offset, (uint32_t)(offset >> 32)), d.seed0, d.seed1);
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu) >= d.cut ? v[i] * d.scale : 0.f;
}

}  // namespace sagnn
