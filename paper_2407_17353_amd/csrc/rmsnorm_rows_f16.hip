// RMS norm kernels for F16 inputs.
#include "rmsnorm_rows.h"

namespace scalify {

template <int WPR, bool RANGE>
static void fwd(const RmsParams& p, hipStream_t s) {
  const int64_t rows = p.block_scale ? (p.R + 63) / 64 * 64 : p.R;
  const dim3 g(rms_grid(rows, WPR, 4)), b(rms_threads(WPR));
  if (p.D == 1024 * WPR) hipLaunchKernelGGL((rms_fwd_rows_kernel<kF16, WPR, true, RANGE>), g, b, 0, s, p);
  else hipLaunchKernelGGL((rms_fwd_rows_kernel<kF16, WPR, false, RANGE>), g, b, 0, s, p);
}

template <bool RANGE>
static void fwd_rows(const RmsParams& p, hipStream_t s) {
  switch (rms_wpr(p.D)) {
    case 1: fwd<1, RANGE>(p, s); break;
    case 2: fwd<2, RANGE>(p, s); break;
    case 4: fwd<4, RANGE>(p, s); break;
    default: fwd<8, RANGE>(p, s); break;
  }
}

template <>
void launch_rms_fwd_rows<kF16>(const RmsParams& p, hipStream_t s) {
  if (rms_ranged(p)) fwd_rows<true>(p, s);
  else fwd_rows<false>(p, s);
}

template <int DYF, int WPR>
static void bwd(const RmsParams& p, hipStream_t s) {
  const dim3 g(rms_bwd_grid(p)), b(rms_threads(WPR));
  if (p.D == 1024 * WPR) hipLaunchKernelGGL((rms_bwd_rows_kernel<kF16, DYF, WPR, true>), g, b, 0, s, p);
  else hipLaunchKernelGGL((rms_bwd_rows_kernel<kF16, DYF, WPR, false>), g, b, 0, s, p);
  if (p.mode == 1) {
    const dim3 t((p.D + LN_TILE_COLS - 1) / LN_TILE_COLS, (unsigned)((p.R + RMS_TILE_ROWS - 1) / RMS_TILE_ROWS));
    hipLaunchKernelGGL((rms_bwd_apply_kernel<kF16, DYF>), t, dim3(LN_TILE_THREADS), 0, s, p);
  }
}

template <int DYF>
static void bwd_dy(const RmsParams& p, hipStream_t s) {
  switch (rms_wpr(p.D)) {
    case 1: bwd<DYF, 1>(p, s); break;
    case 2: bwd<DYF, 2>(p, s); break;
    case 4: bwd<DYF, 4>(p, s); break;
    default: bwd<DYF, 8>(p, s); break;
  }
}

template <>
void launch_rms_bwd_rows<kF16>(const RmsParams& p, hipStream_t s) {
  if (p.dy_fmt == kF16) bwd_dy<kF16>(p, s);
  else if (p.dy_fmt == kF32) bwd_dy<kF32>(p, s);
  else bwd_dy<kE4M3>(p, s);
}

}  // namespace scalify
