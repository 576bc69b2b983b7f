// The products of xent.h: bfloat16 tensors.
#include "xent.h"

namespace sagnn {
int xent_bf16(const XentArgs& a, int tile, bool trans_w, hipStream_t s) { return xent_small<__bf16, SAGNN_GEMM_BF16, 64>(a, tile, trans_w, s); }
}  // namespace sagnn
