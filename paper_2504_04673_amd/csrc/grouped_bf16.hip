// The grouped products of grouped.h and grouped_direct.h: bfloat16 tensors.
#include "grouped_direct.h"

namespace sagnn {
int grouped_bf16(const GroupedArgs& a, int tile, bool trans_w, int64_t blocks, hipStream_t s) {
  if (tile == kDirect256) {
    return grouped_launches(a, blocks, 512, [&](const GroupedArgs& part, dim3 grid) {
      if (trans_w) grouped_direct_kernel<true, 4, 4, 2><<<grid, 512, 0, s>>>(part);
      else grouped_direct_kernel<false, 4, 4, 2><<<grid, 512, 0, s>>>(part);
    });
  }
  return trans_w ? grouped_launch<__bf16, SAGNN_GEMM_BF16, 64, true>(a, tile, blocks, s)
                 : grouped_launch<__bf16, SAGNN_GEMM_BF16, 64, false>(a, tile, blocks, s);
}
int grouped_tn_bf16(const GroupedArgs& a, int tile, int64_t blocks, hipStream_t s) {
  if (tile == kDirect256) {
    return grouped_launches(a, blocks, 512, [&](const GroupedArgs& part, dim3 grid) { grouped_direct_tn_kernel<4, 4, 2><<<grid, 512, 0, s>>>(part); });
  }
  return grouped_tn_launch<__bf16, SAGNN_GEMM_BF16, 64>(a, tile, blocks, s);
}
int grouped_bwd_bf16(const GroupedArgs& rows, int64_t rows_blocks, const GroupedArgs& tn, int64_t tn_blocks, hipStream_t s) {
  grouped_direct_bwd_kernel<4, 4, 2><<<dim3((uint32_t)(rows_blocks + tn_blocks)), 512, 0, s>>>(rows, tn, (int32_t)tn_blocks);
  SAGNN_LAUNCH_CHECK();
  return SAGNN_OK;
}
}  // namespace sagnn
