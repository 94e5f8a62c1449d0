// The gradients' products of the losses (loss_gemm.h): dx = dz w and dw = dz^T x.
#include "loss_gemm.h"

namespace scalify {

hipError_t launch_loss_grads(const LossGemm& p, int epi, int grid, hipStream_t s) {
  if (epi == LOSS_DX) {
    if (p.b_fmt == kE4M3) return launch_one(loss_gemm_kernel<false, true, LOSS_DX, 0, kE4M3>, grid, 256, s, p);
    if (p.b_fmt == kE5M2) return launch_one(loss_gemm_kernel<false, true, LOSS_DX, 0, kE5M2>, grid, 256, s, p);
    return launch_one(loss_gemm_kernel<false, true, LOSS_DX, 0>, grid, 256, s, p);
  }
  if (p.mode == 1) {
    if (p.out_fmt == kF16) return launch_one(loss_gemm_kernel<true, true, LOSS_DW, FORM_F32>, grid, 256, s, p);
    return launch_one(loss_gemm_kernel<true, true, LOSS_DW, FORM_STICKY>, grid, 256, s, p);
  }
  if (p.out_fmt == kF16) return launch_one(loss_gemm_kernel<true, true, LOSS_DW, kF16>, grid, 256, s, p);
  if (p.out_fmt == kE4M3) return launch_one(loss_gemm_kernel<true, true, LOSS_DW, kE4M3>, grid, 256, s, p);
  return launch_one(loss_gemm_kernel<true, true, LOSS_DW, kE5M2>, grid, 256, s, p);
}

}  // namespace scalify
