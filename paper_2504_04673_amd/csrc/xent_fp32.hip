// The products of xent.h: fp32 tensors, fp32 instructions.
#include "xent.h"

namespace sagnn {
int xent_fp32(const XentArgs& a, int tile, bool trans_w, hipStream_t s) { return xent_small<float, SAGNN_GEMM_FP32, 32>(a, tile, trans_w, s); }
}  // namespace sagnn
