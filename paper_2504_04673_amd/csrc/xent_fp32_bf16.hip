// The products of xent.h: fp32 tensors, operands rounded to bfloat16.
#include "xent.h"

namespace sagnn {
int xent_fp32_bf16(const XentArgs& a, int tile, bool trans_w, hipStream_t s) { return xent_small<float, SAGNN_GEMM_BF16, 64>(a, tile, trans_w, s); }
}  // namespace sagnn
