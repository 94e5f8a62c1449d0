// Internal interface of the attention kernels (attention_*.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace scalify {

struct AttnParams {
  // [rows][heads * D], rows ld elements apart; formats; scales (NULL = 1)
  const void *q, *k, *v;
  int64_t ldq, ldk, ldv;
  int q_fmt, k_fmt, v_fmt;
  const float *s_q, *s_k, *s_v;
  int64_t rows_q, rows_k, batch;
  int H, Hkv, G, D;          // G = H / Hkv query heads share a key head
  int causal;
  float alpha;
  const int64_t *q_start, *k_start, *k_len;  // or NULL
  int64_t max_q, max_k;      // bounds of a sequence's rows
  uint32_t group0;           // number of the launch's first workgroup (launch_groups)
  void* out;                 // forward: codes; backward: the stored output (F16)
  int64_t ldo;
  int out_fmt;
  float* out_scale;          // (backward: of the stored output, read)
  float* lse;                // [H][rows_q]: written (or NULL) / read
  int sat;
  // forward, keys of a sequence split over `splits` workgroups
  int splits;
  float* part_o;             // [splits][rows_q][H][D] unnormalised
  float2* part_ml;           // [splits][rows_q][H] running maximum and sum
  // backward
  const void* dout;
  int64_t lddo;
  int do_fmt;
  const float* s_do;
  float *delta, *nd2;        // [H][rows_q]: sum dO O, sum dO^2
  float* nv2;                // [Hkv][rows_k]: sum v^2
  void *dq, *dk, *dv;        // codes (no rescale)
  int64_t lddq, lddk, lddv;
  int dq_fmt, dk_fmt, dv_fmt;
  float *dq_scale, *dk_scale, *dv_scale;
  float *dq32, *dk32, *dv32; // dynamic rescale: fp32 gradients [rows][heads * D], else NULL
  int parts;                 // workgroups that share the queries of 128 keys
  float* part;               // parts > 1: their dk and dv, [parts][2][rows_k][Hkv * D], the first in
                             // place of dk32 and dv32
  uint32_t* amax;            // the three statistics
  float* amax_out;           // optional [3]
  int mode, target;
};

constexpr int kAttnMaxD = 128;

// A launch holds less than 2^32 threads in a dimension of its grid: `groups`
// workgroups of 256 go out as launches of 2^23, which leaves a workgroup's XCD what it
// is in one launch, each with the number of its first one. Stops at a launch that is
// refused, and goes by that launch's status alone, not by an error of an earlier call.
constexpr int64_t kLaunchGroups = 1 << 23;
template <typename... Args>
hipError_t launch_groups(void (*kernel)(AttnParams, Args...), int64_t groups, unsigned y, hipStream_t s, AttnParams p, Args... args) {
  for (int64_t g = 0; g < groups; g += kLaunchGroups) {
    const int64_t n = groups - g < kLaunchGroups ? groups - g : kLaunchGroups;
    p.group0 = (uint32_t)g;
    void* a[] = {&p, (void*)&args...};
    const hipError_t e = hipLaunchKernel((const void*)kernel, dim3((unsigned)n, y), dim3(256), a, 0, s);
    if (e != hipSuccess) {
      (void)hipGetLastError();
      return e;
    }
  }
  return hipSuccess;
}

// Splits of a sequence's keys for the forward, 1 where the grid fills the
// device without, and a workgroup's query columns: 32 that its four waves share
// (few queries), or 128.
struct AttnPlan {
  int splits, cols;
};
AttnPlan attention_plan(int64_t batch, int Hkv, int G, int64_t max_q, int64_t max_k);
hipError_t launch_attention_fwd(const AttnParams& p, const AttnPlan& plan, hipStream_t s);
// The backward's `parts`, 1 where the grid fills the device without.
int attention_bwd_parts(int64_t batch, int Hkv, int G, int64_t max_q, int64_t max_k);
hipError_t launch_attention_bwd(const AttnParams& p, hipStream_t s);

}  // namespace scalify
