// The grouped products of grouped.h: fp32 tensors, operands as three bfloat16 terms.
#include "grouped.h"

namespace sagnn {
int grouped_fp32_bf16x3(const GroupedArgs& a, int tile, bool trans_w, int64_t blocks, hipStream_t s) {
  return trans_w ? grouped_launch<float, SAGNN_GEMM_FP32_BF16X3, 32, true>(a, tile, blocks, s) : grouped_launch<float, SAGNN_GEMM_FP32_BF16X3, 32, false>(a, tile, blocks, s);
}
int grouped_tn_fp32_bf16x3(const GroupedArgs& a, int tile, int64_t blocks, hipStream_t s) {
  return grouped_tn_launch<float, SAGNN_GEMM_FP32_BF16X3, 32>(a, tile, blocks, s);
}
}  // namespace sagnn
