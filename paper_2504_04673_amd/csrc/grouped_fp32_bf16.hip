// The grouped products of grouped.h and grouped_staged.h: fp32 tensors, operands rounded to bfloat16.
#include "grouped_staged.h"

namespace sagnn {
int grouped_fp32_bf16(const GroupedArgs& a, int tile, bool trans_w, int64_t blocks, hipStream_t s) {
  if (tile == kStaged256x128) return grouped_staged_launch<SAGNN_GEMM_BF16, 4, 2>(a, trans_w, blocks, s);
  if (tile == kStaged128x256) return grouped_staged_launch<SAGNN_GEMM_BF16, 2, 4>(a, trans_w, blocks, s);
  return trans_w ? grouped_launch<float, SAGNN_GEMM_BF16, 64, true>(a, tile, blocks, s) : grouped_launch<float, SAGNN_GEMM_BF16, 64, false>(a, tile, blocks, s);
}
int grouped_tn_fp32_bf16(const GroupedArgs& a, int tile, int64_t blocks, hipStream_t s) {
  if (tile == kStaged256x128) return grouped_staged_tn_launch<SAGNN_GEMM_BF16, 4, 2>(a, blocks, s);
  if (tile == kStaged128x256) return grouped_staged_tn_launch<SAGNN_GEMM_BF16, 2, 4>(a, blocks, s);
  return grouped_tn_launch<float, SAGNN_GEMM_BF16, 64>(a, tile, blocks, s);
}
}  // namespace sagnn
