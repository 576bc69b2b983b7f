// The products of xent.h: bfloat16 tensors, in large tiles straight into LDS where rows begin on 16 bytes.
#include "grouped_direct.h"
#include "xent.h"

namespace sagnn {
namespace {
template <bool TRB>
struct DirectProduct {
  using S = __bf16;
  static constexpr int WM = 2, WN = 4, TM = 4, TN = 2, kThreads = 512;
  static constexpr int kLds = direct_lds(256, 256, WN) > xent_lds(WM, WN, TM, TN) ? direct_lds(256, 256, WN) : xent_lds(WM, WN, TM, TN);
  static constexpr bool kTransW = !TRB, kTurned = true;
  static __device__ __forceinline__ void run(const XentArgs& a, const S* A, int64_t lda, int rows, const S* B, int cols, int sum, int padded, char* smem, floatx16 (&acc)[TM][TN]) {
    direct_product<false, TRB, WM, WN, TM, TN>(A, lda, rows, B, a.ldw, cols, padded, smem, acc, sum);
  }
};

// Tiles of 256 x 256 over all listed rows.  Bound by the matrix cores (8192 rows, 1024 by 32768 classes: 430 us, 1279 TFLOP/s), by the weights' bytes where rows
// are few (128 rows of 4096 by 131072 classes, P in one term: a step 1394 us, through fp32 and a conversion 2487).
struct WeightTile {
  static constexpr int WM = 2, WN = 4, TM = 4, TN = 2;
};
__global__ __launch_bounds__(512) void xent_weights_kernel(const XentWeightArgs a) {
  using C = WeightTile;
  __shared__ __attribute__((aligned(1024))) char smem[direct_lds(256, 256, C::WN)];
  const int32_t id = xcd_run((int32_t)blockIdx.x, a.row_tiles * a.col_tiles), band = id / (kXentBand * a.col_tiles), in = id - band * kXentBand * a.col_tiles;
  const int32_t high = a.row_tiles - band * kXentBand < kXentBand ? a.row_tiles - band * kXentBand : kXentBand;
  const int32_t r0 = (band * kXentBand + in % high) * 256, c0 = in / high * 256;
  const int32_t count = *a.count;
  const bool other = count == a.m;
  const __bf16 *A = reinterpret_cast<const __bf16*>(other ? a.A2 : a.A) + r0, *B = reinterpret_cast<const __bf16*>(other ? a.B2 : a.B) + c0;
  const int64_t lda = other ? a.lda2 : a.lda, ldb = other ? a.ldb2 : a.ldb;
  const int rows = a.rows - r0 < 256 ? a.rows - r0 : 256, cols = a.cols - c0 < 256 ? a.cols - c0 : 256;
  floatx16 acc[C::TM][C::TN];
  // (whole eights of a row are loaded: what is behind a width is zeros, or a result's that is not stored)
  direct_product<true, true, C::WM, C::WN, C::TM, C::TN>(A, lda, (rows + 7) & ~7, B, ldb, (cols + 7) & ~7, count < a.m ? count : a.m, smem, acc);
  __syncthreads();
  __bf16* out = reinterpret_cast<__bf16*>(a.out) + (int64_t)r0 * a.ldo + c0;
  const float scale = count > 0 ? a.scale : 0.f;              // (no rows: zeros, whatever it is)
  if (a.wide) {
#pragma unroll
    for (int i = 0; i < C::TM * C::TN * 4; ++i) {
      const int tm = i / (C::TN * 4), tn = i / 4 % C::TN, v = i % 4 * 4;
      const float y[4] = {acc[tm][tn][v] * scale, acc[tm][tn][v + 1] * scale, acc[tm][tn][v + 2] * scale, acc[tm][tn][v + 3] * scale};
      Turn<C>::put(smem, tm, tn, v, y);
    }
    Turn<C>::store(smem, out, rows, cols, [&](int r) { return r * a.ldo; });
    return;
  }
  tile_fours<C::WM, C::WN, C::TM, C::TN>(acc, [&](int r, int c, float (&y)[4]) {
    if (r >= rows) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] *= scale;
    store_four(out + r * a.ldo + c, y, cols - c);
  });
}
}  // namespace

int xent_weights_bf16(const XentWeightArgs& a, hipStream_t s) {
  xent_weights_kernel<<<dim3((uint32_t)(a.row_tiles * a.col_tiles)), 512, 0, s>>>(a);
  SAGNN_LAUNCH_CHECK();
  return SAGNN_OK;
}

int xent_bf16(const XentArgs& a, int tile, bool trans_w, hipStream_t s) {
  if (tile == kDirect256) return trans_w ? xent_launch<DirectProduct<false>>(a, s) : xent_launch<DirectProduct<true>>(a, s);
  return xent_small<__bf16, SAGNN_GEMM_BF16, 64>(a, tile, trans_w, s);
}
}  // namespace sagnn
