// The products of xent.h: fp32 tensors, operands as three bfloat16 terms.
#include "xent_staged.h"

namespace sagnn {
int xent_fp32_bf16x3(const XentArgs& a, int tile, bool trans_w, hipStream_t s) {
  if (tile == kStaged256x128) return xent_staged<SAGNN_GEMM_FP32_BF16X3, 4, 2>(a, trans_w, s);
  if (tile == kStaged128x256) return xent_staged<SAGNN_GEMM_FP32_BF16X3, 2, 4>(a, trans_w, s);
  return xent_small<float, SAGNN_GEMM_FP32_BF16X3, 32>(a, tile, trans_w, s);
}
}  // namespace sagnn
