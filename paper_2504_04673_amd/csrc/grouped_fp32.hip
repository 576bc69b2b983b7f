// The grouped products of grouped.h: fp32 instructions.
#include "grouped.h"

namespace sagnn {
int grouped_fp32(const GroupedArgs& a, int tile, bool trans_w, int64_t blocks, hipStream_t s) {
  return trans_w ? grouped_launch<float, SAGNN_GEMM_FP32, 32, true>(a, tile, blocks, s) : grouped_launch<float, SAGNN_GEMM_FP32, 32, false>(a, tile, blocks, s);
}
int grouped_tn_fp32(const GroupedArgs& a, int tile, int64_t blocks, hipStream_t s) {
  return grouped_tn_launch<float, SAGNN_GEMM_FP32, 32>(a, tile, blocks, s);
}
}  // namespace sagnn
