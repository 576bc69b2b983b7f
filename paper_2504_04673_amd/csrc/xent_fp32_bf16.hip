// The products of xent.h: fp32 tensors, operands rounded to bfloat16.
#include "xent_staged.h"

namespace sagnn {
int xent_fp32_bf16(const XentArgs& a, int tile, bool trans_w, hipStream_t s) {
  if (tile == kStaged256x128) return xent_staged<SAGNN_GEMM_BF16, 4, 2>(a, trans_w, s);
  if (tile == kStaged128x256) return xent_staged<SAGNN_GEMM_BF16, 2, 4>(a, trans_w, s);
  return xent_small<float, SAGNN_GEMM_BF16, 64>(a, tile, trans_w, s);
}
}  // namespace sagnn
