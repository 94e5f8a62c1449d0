// Internal interface of the RMS norm kernels (rmsnorm_*.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace scalify {

// Rows of D <= 8192 values, row-major.
struct RmsParams {
  const void* x;        // [R][ldx], format x_fmt: the branch, or (backward) the stored sum
  int64_t ldx;
  int x_fmt;
  const float* s_x;     // scales (NULL = 1)
  int has_res;          // (an array without elements may have no data)
  const void* res;      // forward: residual [R][ldr]; backward: the gradient that reaches the sum itself
  int64_t ldr;
  int res_fmt;
  const float* s_res;
  const void* dy;       // backward: [R][lddy], format dy_fmt
  int64_t lddy;
  int dy_fmt;
  const float* s_dy;
  const float* gamma;   // [D] or NULL (1)
  void* sum;            // forward: optional stored sum [R][lds]
  int64_t lds;
  int sum_fmt;
  float* sum_scale;
  void* out;            // forward y / backward dx codes [R][ldo]
  int64_t ldo;
  int out_fmt;
  float* out_scale;
  float* row_scale;     // forward: optional [R]
  uint8_t* block_scale; // forward: optional packed MX bytes
  float* pre_out;       // optional fp32 [R][D]: the values before the rescale and cast
  int64_t R;
  int D;
  float eps;
  int sat, target, mode;  // backward rescale: mode 1 = amax, 0 = none
  uint32_t* hdr;        // backward: workspace header, and the call's tag in it (stat_header.h)
  uint64_t tag;
  float* partial;       // backward: per-row numbers [R][4], then partial dgamma [workgroups][stride]
  float* amax_out;      // backward: optional
  float* dgamma;        // backward: optional [D]
};

// The backward's row kernel: at most this many workgroups (its partial dgamma
// rows are counted into the workspace before the device is known).
constexpr int kRmsMaxGroups = 1024;
inline int rms_wpr(int64_t D) { return D <= 1024 ? 1 : (D <= 2048 ? 2 : (D <= 4096 ? 4 : 8)); }  // waves of a row
int rms_grid(int64_t R, int wpr, int waves);    // workgroups that keep `waves` waves on every SIMD
int64_t rmsnorm_groups(int64_t R, int64_t D);   // workgroups that R rows of D can use, at most kRmsMaxGroups
int64_t rmsnorm_ws_floats(int64_t R, int64_t D);
int rms_bwd_grid(const RmsParams& p);           // those launched on the current device
hipError_t launch_rmsnorm_fwd(const RmsParams& p, hipStream_t s);
hipError_t launch_rmsnorm_bwd(const RmsParams& p, hipStream_t s);

// One source file for each class of x's element size (kE4M3: the 8-bit formats).
template <int XF>
void launch_rms_fwd_rows(const RmsParams& p, hipStream_t s);
template <int XF>
void launch_rms_bwd_rows(const RmsParams& p, hipStream_t s);

}  // namespace scalify
