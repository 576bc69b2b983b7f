// The products of xent.h in the large tiles of fp32 tensors on the bfloat16 matrix cores.
#pragma once
#include "grouped_staged.h"
#include "xent.h"

namespace sagnn {

template <int PREC, bool TRB, int WM_, int WN_, bool LONG>
struct StagedProduct {
  using S = float;
  static constexpr int WM = WM_, WN = WN_, TM = 2, TN = 2, kThreads = WM * WN * 64;
  static constexpr int kOperands = 2 * (StagedOperand<PREC, false, WM * 64, kThreads>::kBytes + StagedOperand<PREC, TRB, WN * 64, kThreads>::kBytes);
  static constexpr int kLds = kOperands > xent_lds(WM, WN, TM, TN) ? kOperands : xent_lds(WM, WN, TM, TN);
  static constexpr bool kTransW = !TRB, kTurned = false;
  static __device__ __forceinline__ void run(const XentArgs& a, const S* A, int64_t lda, int rows, const S* B, int cols, int sum, int, char* smem, floatx16 (&acc)[TM][TN]) {
    staged_product<PREC, false, TRB, WM, WN, TM, TN, LONG>(A, lda, rows, B, a.ldw, cols, sum, smem, acc, a.run);
  }
};

template <int PREC, int WM, int WN>
int xent_staged(const XentArgs& a, bool trans_w, hipStream_t s) {
  const bool several = a.share > a.run;
  if (trans_w) return several ? xent_launch<StagedProduct<PREC, false, WM, WN, true>>(a, s) : xent_launch<StagedProduct<PREC, false, WM, WN, false>>(a, s);
  return several ? xent_launch<StagedProduct<PREC, true, WM, WN, true>>(a, s) : xent_launch<StagedProduct<PREC, true, WM, WN, false>>(a, s);
}

}  // namespace sagnn
