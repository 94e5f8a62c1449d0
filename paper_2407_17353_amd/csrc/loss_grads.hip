// The gradients' products of the losses (loss_gemm.h): dx = dz w and dw = dz^T x.
#include "loss_gemm.h"

namespace scalify {

hipError_t launch_loss_grads(const LossGemm& p, int epi, int grid, hipStream_t s) {
  if (epi == LOSS_DX) return launch_one(loss_gemm_kernel<false, true, LOSS_DX>, grid, 256, s, p);
  return launch_one(loss_gemm_kernel<true, true, LOSS_DW>, grid, 256, s, p);
}

}  // namespace scalify
