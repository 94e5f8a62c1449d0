// The logits' products of the losses (loss_gemm.h): both operands along k.
#include "loss_gemm.h"

namespace scalify {

template <int EPI>
static hipError_t launch_rows_of(const LossGemm& p, int grid, hipStream_t s) {
  if (p.b_fmt == kE4M3) return launch_one(loss_gemm_kernel<false, false, EPI, 0, kE4M3>, grid, 256, s, p);
  if (p.b_fmt == kE5M2) return launch_one(loss_gemm_kernel<false, false, EPI, 0, kE5M2>, grid, 256, s, p);
  return launch_one(loss_gemm_kernel<false, false, EPI, 0>, grid, 256, s, p);
}

hipError_t launch_loss_logits(const LossGemm& p, int epi, int grid, hipStream_t s) {
  if (epi == LOSS_STATS) return launch_rows_of<LOSS_STATS>(p, grid, s);
  if (epi == LOSS_PICK) return launch_rows_of<LOSS_PICK>(p, grid, s);
  return launch_rows_of<LOSS_DZ>(p, grid, s);
}

}  // namespace scalify
