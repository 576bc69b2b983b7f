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
}  // namespace

int xent_bf16(const XentArgs& a, int tile, bool trans_w, hipStream_t s) {
  if (tile == kDirect256) return trans_w ? xent_launch<DirectProduct<false>>(a, s) : xent_launch<DirectProduct<true>>(a, s);
  return xent_small<__bf16, SAGNN_GEMM_BF16, 64>(a, tile, trans_w, s);
}
}  // namespace sagnn
