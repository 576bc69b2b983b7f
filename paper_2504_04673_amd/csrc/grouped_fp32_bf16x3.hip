// The grouped products of grouped.h and grouped_staged.h: fp32 tensors, operands as three bfloat16 terms.
#include "grouped_staged.h"

namespace sagnn {
int grouped_fp32_bf16x3(const GroupedArgs& a, int tile, bool trans_w, int64_t blocks, hipStream_t s) {
  if (tile == kStaged256x128) return grouped_staged_launch<SAGNN_GEMM_FP32_BF16X3, 4, 2>(a, trans_w, blocks, s);
  if (tile == kStaged128x256) return grouped_staged_launch<SAGNN_GEMM_FP32_BF16X3, 2, 4>(a, trans_w, blocks, s);
  return trans_w ? grouped_launch<float, SAGNN_GEMM_FP32_BF16X3, 32, true>(a, tile, blocks, s) : grouped_launch<float, SAGNN_GEMM_FP32_BF16X3, 32, false>(a, tile, blocks, s);
}
int grouped_tn_fp32_bf16x3(const GroupedArgs& a, int tile, int64_t blocks, hipStream_t s) {
  if (tile == kStaged256x128) return grouped_staged_tn_launch<SAGNN_GEMM_FP32_BF16X3, 4, 2>(a, blocks, s);
  if (tile == kStaged128x256) return grouped_staged_tn_launch<SAGNN_GEMM_FP32_BF16X3, 2, 4>(a, blocks, s);
  return grouped_tn_launch<float, SAGNN_GEMM_FP32_BF16X3, 32>(a, tile, blocks, s);
}
}  // namespace sagnn
