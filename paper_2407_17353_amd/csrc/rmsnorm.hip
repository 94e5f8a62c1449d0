// RMS norm: launches, and the kernel that ends a backward call.
#include "kernels.h"
#include "rmsnorm_rows.h"

namespace scalify {

// The end of a backward call: dgamma[j] = the workgroups' partial sums in a
// fixed order (16 waves sum interleaved shares, then a fixed tree), and, once
// no kernel of the call reads an input scale any more (dx's may be the same
// memory), the output scale and the statistic.
constexpr int RMS_PARAM_WAVES = 16;

__global__ __launch_bounds__(64 * RMS_PARAM_WAVES) void rms_bwd_end_kernel(RmsParams p, int groups) {
  __shared__ float red[RMS_PARAM_WAVES][64];
  const int c = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int j = blockIdx.x * 64 + c;
  const int64_t dp = layernorm_param_stride(p.D);
  const float* part = p.partial + 4 * p.R;
  float g = 0.0f;
  if (p.dgamma && j < p.D) {
#pragma unroll 8
    for (int k = w; k < groups; k += RMS_PARAM_WAVES) g += part[(int64_t)k * dp + j];
  }
  red[w][c] = g;
  __syncthreads();
  if (w == 0 && p.dgamma && j < p.D) {
    float s[RMS_PARAM_WAVES];
#pragma unroll
    for (int i = 0; i < RMS_PARAM_WAVES; ++i) s[i] = red[i][c];
#pragma unroll
    for (int h = 1; h < RMS_PARAM_WAVES; h *= 2)
#pragma unroll
      for (int i = 0; i < RMS_PARAM_WAVES; i += 2 * h) s[i] += s[i + h];
    p.dgamma[j] = s[0];
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    const uint32_t amax = p.R > 0 ? p.hdr[0] : 0u;  // (without rows no kernel opened the header)
    const int e_r = p.mode == 1 ? rescale_exponent(amax, p.target) : 0;
    *p.out_scale = pow2_float(clamp_e8m0(rms_exps(p).e + e_r));
    if (p.amax_out) *p.amax_out = __uint_as_float(amax);
    if (p.R > 0) stat_retire(p.hdr);
  }
}

int64_t rmsnorm_groups(int64_t R, int64_t D) {
  const int64_t rpw = rms_rpw(rms_wpr(D));
  const int64_t need = (R + rpw - 1) / rpw;
  return need < kRmsMaxGroups ? need : kRmsMaxGroups;
}

int64_t rmsnorm_ws_floats(int64_t R, int64_t D) {
  return 4 * R + rmsnorm_groups(R, D) * layernorm_param_stride(D);
}

int rms_grid(int64_t R, int wpr, int waves) {
  const int rpw = rms_rpw(wpr);
  const int64_t need = (R + rpw - 1) / rpw;
  const int64_t g = (int64_t)(wpr == 8 ? waves / 2 : waves) * gemm4_grid(1 << 30);  // (CUs of the current device)
  return (int)(need < 1 ? 1 : (need < g ? need : g));
}

// Within the workspace's partial rows. (512 workgroups: with 1024 the partial rows of
// dgamma cost more than the further loads in flight bring, 134 us for 123 at 16384 x
// 4096, with 256 too few loads are in flight, 195 us.)
int rms_bwd_grid(const RmsParams& p) {
  const int g = rms_grid(p.R, rms_wpr(p.D), 2);
  const int64_t most = rmsnorm_groups(p.R, p.D);
  return g < most ? g : (int)most;
}

__global__ void rms_fwd_empty_kernel(RmsParams p) {
  *p.out_scale = 1.0f;
  if (p.sum_scale) *p.sum_scale = pow2_float(clamp_e8m0(max(pow2_exponent(p.s_x), pow2_exponent(p.s_res))));
}

hipError_t launch_rmsnorm_fwd(const RmsParams& p, hipStream_t s) {
  if (p.R == 0) hipLaunchKernelGGL(rms_fwd_empty_kernel, dim3(1), dim3(1), 0, s, p);
  else if (p.x_fmt == kF16) launch_rms_fwd_rows<kF16>(p, s);
  else if (p.x_fmt == kF32) launch_rms_fwd_rows<kF32>(p, s);
  else launch_rms_fwd_rows<kE4M3>(p, s);
  return hipGetLastError();
}

hipError_t launch_rmsnorm_bwd(const RmsParams& p, hipStream_t s) {
  int groups = 0;
  if (p.R > 0) {
    groups = rms_bwd_grid(p);
    if (p.x_fmt == kF16) launch_rms_bwd_rows<kF16>(p, s);
    else if (p.x_fmt == kF32) launch_rms_bwd_rows<kF32>(p, s);
    else launch_rms_bwd_rows<kE4M3>(p, s);
  }
  const int cols = p.dgamma ? (p.D + 63) / 64 : 0;
  hipLaunchKernelGGL(rms_bwd_end_kernel, dim3(cols < 1 ? 1 : cols), dim3(64 * RMS_PARAM_WAVES), 0, s, p, groups);
  return hipGetLastError();
}

}  // namespace scalify
