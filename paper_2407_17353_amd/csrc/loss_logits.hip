// The logits' products of the losses (loss_gemm.h): both operands along k.
#include "loss_gemm.h"

namespace scalify {

hipError_t launch_loss_logits(const LossGemm& p, int epi, int grid, hipStream_t s) {
  if (epi == LOSS_STATS) return launch_one(loss_gemm_kernel<false, false, LOSS_STATS, 0>, grid, 256, s, p);
  if (epi == LOSS_PICK) return launch_one(loss_gemm_kernel<false, false, LOSS_PICK, 0>, grid, 256, s, p);
  return launch_one(loss_gemm_kernel<false, false, LOSS_DZ, 0>, grid, 256, s, p);
}

}  // namespace scalify
