// Device helpers of the losses' kernels.
#pragma once
#include "attention_dev.h"
#include "loss.h"

namespace scalify {

// Factor of a row's logits in base 2; past [2^-100, 2^64] it gives equal logits, or the
// largest alone.
__device__ __forceinline__ float logit_factor(const LossParams& p, int64_t row) {
  const int e = pow2_exponent(p.s_x) + pow2_exponent(p.s_w) + (p.row_scale ? pow2_exponent(p.row_scale + row) : 0);
  const float f = ldexpf(kLog2e / p.temp, e < -200 ? -200 : (e > 200 ? 200 : e));
  return fminf(fmaxf(f, 0x1p-100f), 0x1p64f);
}

// Four values times inv = 2^-shift, inside the conversions' window, to F16 (round to nearest
// even; the product is exact unless F16 overflows or is 0), two a word. NAN: some may be.
template <bool NAN_>
__device__ __forceinline__ u2 codes4_f16(const float* y, float inv, bool sat) {
  u2 w;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float a = y[2 * i] * inv, b = y[2 * i + 1] * inv;
    if (sat) {
      a = __builtin_amdgcn_fmed3f(a, -65504.0f, 65504.0f);
      b = __builtin_amdgcn_fmed3f(b, -65504.0f, 65504.0f);
    }
    asm("v_cvt_pk_f16_f32 %0, %1, %2" : "=v"(w[i]) : "v"(a), "v"(b));
    if constexpr (NAN_) {
      uint32_t lo = w[i] & 0xFFFFu, hi = w[i] >> 16;
      if (y[2 * i] != y[2 * i]) lo = FmtTraits<kF16>::NANC | ((__float_as_uint(y[2 * i]) >> 16) & 0x8000u);
      if (y[2 * i + 1] != y[2 * i + 1]) hi = FmtTraits<kF16>::NANC | ((__float_as_uint(y[2 * i + 1]) >> 16) & 0x8000u);
      w[i] = lo | (hi << 16);
    }
  }
  return w;
}
// The same to an 8-bit format, scale = 2^shift.
template <int F, bool NAN_>
__device__ __forceinline__ uint32_t codes4_fp8(const float* y, float scale, bool sat) {
  uint32_t w = cast4_fp8_hw<F>(__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3]), scale, sat);
  if constexpr (NAN_) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (y[i] != y[i]) {
        const uint32_t c = FmtTraits<F>::NANC | ((__float_as_uint(y[i]) >> 24) & 0x80u);
        w = (w & ~(0xFFu << (8 * i))) | (c << (8 * i));
      }
  }
  return w;
}
// A statistic is raised to `a`. Most are below it already, and one read is cheaper than an
// atomic on the word that all share (8192 of them: 80 us); a read that is late is too low.
__device__ __forceinline__ void raise_amax(uint32_t* word, float a) {
  const uint32_t u = __float_as_uint(a);
  if (a > 0.f && u > __hip_atomic_load(word, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) atomicMax(word, u);
}
// A sum's terms 2^(x f - m2) are taken with one rounding, that of x f left out; it may come to
// half a step of m2, the rounded largest x f, which m2 + log2(sum) so makes good. From here on
// that could end fp32's exponents: such a row's differences are formed first.
constexpr float kLargeLogit = 0x1p28f;
__device__ __forceinline__ bool is_large(float m2) { return fabsf(m2) >= kLargeLogit; }

// A probability 2^(z - l) is at most 1, but l has the roundings of a stored log-sum-exp, 2^-22 of
// it in all: from here on dz is held to that (F16 would end at 2; a NaN stays).
constexpr float kLargeSum = 0x1p20f;
__device__ __forceinline__ float held_log(float arg, float l) { return fabsf(l) >= kLargeSum && arg > 0.f ? 0.f : arg; }

// (m, n) and (mo, no), maxima (base 2; -Inf where there is nothing) and sums, as one. A NaN
// is in the sums.
__device__ __forceinline__ void join_sums(float& m, float& n, float mo, float no) {
  const float t = fmaxf(m, mo);
  const float a = m == -__builtin_inff() ? 0.f : n * exp2f(m - t);
  const float c = mo == -__builtin_inff() ? 0.f : no * exp2f(mo - t);
  n = a + c;
  m = t;
}

__device__ __forceinline__ float wave_max(float v) {
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}
__device__ __forceinline__ int wave_max(int v) {
  for (int o = 32; o > 0; o >>= 1) v = max(v, __shfl_xor(v, o, 64));
  return v;
}

__device__ __forceinline__ int hdr_exponent(const uint32_t* hdr, int word) {
  return hdr[word] == 0u ? 0 : floor_log2_bits(hdr[word]);
}

// Exponent of a row's weight in dw, biased; 0 where g (times T) is 0 or not finite. r: its row
// scale.
__device__ __forceinline__ int row_weight(float g, float r) {
  const uint32_t a = __float_as_uint(fabsf(g));
  const int w = floor_log2_bits(a) + pow2_exponent(&r) + kWeightBias;
  return a == 0u || a >= 0x7F800000u ? 0 : w;
}
// The powers of two of such a row: out of dz, and on x for dw. most: the largest row_weight.
// (Rows whose g is 0 or not finite keep x.)
struct RowUnit {
  int dz, x;
};
__device__ __forceinline__ RowUnit row_unit(float g, float r, int most, int ec) {
  const int w = row_weight(g, r);
  if (w == 0) return {ec, 0};
  const int below = most - w, share = min(below, kLossShare);
  return {floor_log2_bits(__float_as_uint(fabsf(g))) + share, share - below};
}
// Unit of dw's products less that of dz.
__device__ __forceinline__ int hdr_weight(const uint32_t* hdr) { return hdr[LOSS_WEIGHT] == 0u ? 0 : (int)hdr[LOSS_WEIGHT] - kWeightBias; }

// Unit of the products: a gradient's data in its propagated scale is the product times
// 2^unit.
__device__ __forceinline__ int unit_of(const LossParams& p, bool dw) {
  return (dw ? hdr_weight(p.hdr) : hdr_exponent(p.hdr, LOSS_CMAX)) - kLossGradLog2;
}
__device__ __forceinline__ int base_of(const LossParams& p, bool dw) { return pow2_exponent(p.s_dloss) + pow2_exponent(dw ? p.s_x : p.s_w); }
__device__ __forceinline__ int out_exponent(const LossParams& p, bool dw, int base, int unit) {
  const uint32_t a = p.hdr[dw ? LOSS_AMAX_DW : LOSS_AMAX_DX];
  const bool plain = p.mode != 1 || a == 0u || a >= 0x7F800000u;
  return clamp_e8m0(base + (plain ? 0 : floor_log2_bits(a) + unit - p.target));
}

template <int F>
__device__ __forceinline__ void store_codes(void* out, int64_t e, const uint32_t (&u)[16], int cols, int shift, bool sat) {
  const bool fast = shift >= kFastShiftMinSub && shift <= kFastShiftMax;
  uint32_t w[8];
  encode16<F>(u, shift, fast ? pow2_float(shift) : 1.0f, fast, sat, w);
  if (cols >= 16) {
    store_words16<F>(out, e, w);
  } else {
#pragma unroll
    for (int i = 0; i < 15; ++i)
      if (i < cols) store1<F>(out, e + i, word_code<F>(w, i));
  }
}

}  // namespace scalify
