// RMS norm with the residual's addition, forward and backward, each row read
// once.
//
//   h = x 2^(e_x - e_h) + r 2^(e_r - e_h), stored as sum; the stored value is normalised
//   inv = 1 / sqrt(mean h^2 + eps),  y = h inv gamma
//   g = dy gamma,  c = inv^2 mean(g h),  dx = inv (g - h c)  [+ the sum's own gradient]
//
// What bounds them: HBM. Forward: x and r read, sum and out written. A lane holds
// one chunk of 16 columns, so a row of up to 1024 columns belongs to one wave, of
// up to 2048 to two, 4096 to four, 8192 to eight (WPR), and the next row's codes
// are loaded while a row is computed. (Two chunks a lane, as the LayerNorm's
// kernels hold, spilled here: the backward keeps h, dy, gamma and dgamma's partial
// sums at once.) Both sums of the backward (h^2 and g h) are taken in one pass, so
// a row needs one exchange between its waves. 16384 x 4096: forward with F16 input,
// residual and sum and E4M3 output with MX scales 95 us (4.9 TB/s), backward with F16
// throughout 122 us (4.4 TB/s); 8 x 4096, forward, 5 us. What a width leaves of its
// waves without columns counts against it: F16 to E4M3 with row scales and no residual,
// 16384 x 4096 takes 38 us (5.4 TB/s), 16384 x 5120, five of eight waves, 74 (3.4),
// 131072 x 512, half of a wave, 68 (3.0) and 524288 x 128, 8 lanes of 64, 257 (0.8).
//
// 8-bit formats are one class of the templates (element size decides the loads);
// which of the two it is, and every other tensor's format, is a uniform branch.
#pragma once
#include "layernorm_rows.h"
#include "rmsnorm.h"

namespace scalify {

// A format's class: what the loads depend on.
__host__ __device__ constexpr int fmt_class(int f) { return f == kE5M2 ? kE4M3 : f; }

template <int CLS>
__device__ __forceinline__ void rms_decode16(int fmt, const uint32_t* w, float (&x)[16]) {
  if constexpr (CLS == kE4M3) {
    if (fmt == kE5M2) ln_decode16<kE5M2>(w, x);
    else ln_decode16<kE4M3>(w, x);
  } else {
    ln_decode16<CLS>(w, x);
  }
}

// Raw codes of a tensor of 8 or 16 bits whose class is not a template parameter.
__device__ __forceinline__ void rms_load_any(int fmt, const void* base, int64_t e, int valid, uint32_t (&w)[8]) {
  if (fmt == kF16) {
    ln_load_raw<kF16>(base, e, valid, w);
  } else {
    uint32_t b[4];
    ln_load_raw<kE4M3>(base, e, valid, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = b[i];
  }
}

__device__ __forceinline__ void rms_decode_any(int fmt, const uint32_t* w, float (&x)[16]) {
  if (fmt == kF16) ln_decode16<kF16>(w, x);
  else rms_decode16<kE4M3>(fmt, w, x);
}

// Cast and store 16 values times 2^-shift at column n of a row, any output format.
__device__ __forceinline__ void rms_store_any(int fmt, void* out, int64_t off, int valid, const float (&y)[16],
                                              int shift, bool sat) {
  const bool fast = shift >= kFastShiftMinSub && shift <= kFastShiftMax;
  const float scale = fast ? pow2_float(shift) : 1.0f;
  if (fmt == kF16) ln_store16<kF16>(out, off, valid, y, shift, scale, fast, sat);
  else if (fmt == kE4M3) ln_store16<kE4M3>(out, off, valid, y, shift, scale, fast, sat);
  else ln_store16<kE5M2>(out, off, valid, y, shift, scale, fast, sat);
}

// Cast to the sum's format, store, and read back what was stored.
template <int F>
__device__ __forceinline__ void rms_store_sum(void* sum, int64_t off, int valid, bool store, float (&h)[16], bool sat) {
  uint32_t u[16], w[8];
#pragma unroll
  for (int i = 0; i < 16; ++i) u[i] = __float_as_uint(h[i]);
  encode16<F>(u, 0, 1.0f, true, sat, w);
  if (store) {
    if (valid >= 16) {
      store_words16<F>(sum, off, w);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (i < valid) store1<F>(sum, off + i, word_code<F>(w, i));
    }
  }
  ln_decode16<F>(w, h);
}

// Whether the rows of a forward call may hold any magnitude: FP32 ones, and the sum
// of a residual that no 16- or 8-bit array takes up (its parts lie on scales that may be
// far apart, and where the larger one's is 0 the other is what is normalised: 16384 x
// 4096 with row scales 68 us, 65 without the division).
inline bool rms_ranged(const RmsParams& p) { return p.x_fmt == kF32 || (p.has_res && !p.sum); }

// 1 / sqrt(ss / D + eps) of a row, 0 where that is 1 / 0. Rows that may hold any
// magnitude (RANGE) are first divided by the power of two 2^k of their
// largest one, so that no square leaves the range, ss is that of the divided
// row, and so is the result (rms(h) = 2^k rms(h / 2^k)); in 64 bits, since
// eps / 2^2k may be any size. (Of 16- and 8-bit data, stored sums among them, no
// square or sum of squares leaves the fp32 range.)
template <bool RANGE>
__device__ __forceinline__ float rms_inv(float ss, int D, float eps, int k) {
  if constexpr (RANGE) {
    const double m = (double)(ss / (float)D) + ldexp((double)eps, -2 * k);
    return m > 0.0 ? (float)(1.0 / sqrt(m)) : (m == 0.0 ? 0.0f : __builtin_nanf(""));
  } else {
    const float m = ss / (float)D + eps;
    return m == 0.0f ? 0.0f : 1.0f / sqrtf(m);
  }
}

// Maximum over the wave, then over the waves of a row.
__device__ __forceinline__ float wave_max(float a) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) a = fmaxf(a, __shfl_xor(a, off, 64));
  return a;
}
template <int WPR>
__device__ __forceinline__ float row_max(float a, float (*slot)[WPR], int row, int part, int lane) {
  a = wave_max(a);
  if constexpr (WPR > 1) {
    if (lane == 0) slot[row][part] = a;
    __syncthreads();
    a = slot[row][0];
#pragma unroll
    for (int k = 1; k < WPR; ++k) a = fmaxf(a, slot[row][k]);
  }
  return a;
}

// The row divided by the power of two of its largest magnitude; returns its exponent. Not
// below 2^-100: the squares of the smallest numbers, 2^-149, then lie over 2^-98, and the
// divided row's 1 / rms, which eps alone may give (2^-100 / sqrt(eps)), is a normal number.
template <int WPR>
__device__ __forceinline__ int rms_range(float (&h)[16], float (*slot)[WPR], int row, int part, int lane) {
  float a = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) a = fmaxf(a, fabsf(h[i]));
  const int k = max(rescale_exponent(__float_as_uint(row_max<WPR>(a, slot, row, part, lane)), 0), -100);
#pragma unroll
  for (int i = 0; i < 16; ++i) h[i] = __builtin_ldexpf(h[i], -k);
  return k;
}

// Threads of a workgroup and its rows at a time: 4 waves, or the 8 of a wide row.
__host__ __device__ constexpr int rms_threads(int wpr) { return wpr == 8 ? 512 : 256; }
__host__ __device__ constexpr int rms_rpw(int wpr) { return wpr == 8 ? 1 : 4 / wpr; }

// Byte of row r and 32-column block b in the packed order of the block-scaled
// matmul (words of four rows 16 apart).
__device__ __forceinline__ int64_t mx_byte(int64_t r, int b, int64_t groups) {
  const int64_t word = ((int64_t)(b >> 2) * groups + (r >> 6)) * 64 + 16 * (b & 3) + (r & 15);
  return 4 * word + ((r >> 4) & 3);
}

// RANGE: of rows of any magnitude (rms_ranged).
template <int XF, int WPR, bool FULL, bool RANGE>
__global__ __launch_bounds__(rms_threads(WPR)) void rms_fwd_rows_kernel(RmsParams p) {
#pragma clang fp contract(off)
  constexpr int RPW = rms_rpw(WPR);
  __shared__ float s1[2][RPW][WPR][1], sm[2][RPW][WPR], sr[2][RPW][WPR];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int slot = wave / WPR, part = wave % WPR;
  const bool sat = p.sat != 0;
  const int n = 16 * (lane + 64 * part), valid = FULL ? 16 : p.D - n;  // (may be <= 0)
  const bool res = p.has_res != 0;
  int dx = 0, dr = 0;
  if (res) {
    const int ex = pow2_exponent(p.s_x), er = pow2_exponent(p.s_res), eh = max(ex, er);
    dx = ex - eh;
    dr = er - eh;
  }
  // Rows are padded to whole groups of 64 where packed scales are written.
  const int64_t groups = (p.R + 63) / 64;
  const int64_t rows = p.block_scale ? groups * 64 : p.R;
  const int64_t stride = (int64_t)gridDim.x * RPW;
  uint32_t w[ln_chunk_words<XF>()], wr[8];
  int64_t r0 = (int64_t)blockIdx.x * RPW;
  auto load = [&](int64_t r) {
    const int v = r < p.R ? valid : 0;
    ln_load_raw<XF>(p.x, r * p.ldx + n, v, w);
    if (res) rms_load_any(p.res_fmt, p.res, r * p.ldr + n, v, wr);
  };
  load(r0 + slot);
  float gam[16];
  ln_param16(p.gamma, n, max(valid, 0), 1.0f, gam);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    // (with a residual the entry point refuses an output scale in the memory of
    // an input scale, which every workgroup reads)
    *p.out_scale = 1.0f;
    if (p.sum_scale) *p.sum_scale = pow2_float(clamp_e8m0(max(pow2_exponent(p.s_x), pow2_exponent(p.s_res))));
  }
  int turn = 0;
#pragma unroll 1
  for (; r0 < rows; r0 += stride, turn ^= 1) {
    const int64_t r = r0 + slot;
    const bool ok = r < p.R;
    float h[16];
    rms_decode16<XF>(p.x_fmt, w, h);
    if (res) {
      float q[16];
      rms_decode_any(p.res_fmt, wr, q);
#pragma unroll
      for (int i = 0; i < 16; ++i) h[i] = __builtin_ldexpf(h[i], dx) + __builtin_ldexpf(q[i], dr);
    }
    load(r + stride);
    if (p.sum) {
      const int64_t off = r * p.lds + n;
      const bool st = ok && (FULL || valid > 0);
      if (p.sum_fmt == kF16) rms_store_sum<kF16>(p.sum, off, valid, st, h, sat);
      else if (p.sum_fmt == kE4M3) rms_store_sum<kE4M3>(p.sum, off, valid, st, h, sat);
      else rms_store_sum<kE5M2>(p.sum, off, valid, st, h, sat);
    }
    // (the two turns' slots alternate: a wave that is a row ahead does not
    // overwrite what its neighbour still reads)
    int k = 0;
    if constexpr (RANGE) k = rms_range<WPR>(h, sr[turn], slot, part, lane);
    float cs = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) cs = fmaf(h[i], h[i], cs);  // columns >= D are 0
    float ss[1] = {wave_sum(cs)};
    row_sum<WPR, 1>(ss, s1[turn], slot, part, lane);
    const float inv = rms_inv<RANGE>(ss[0], p.D, p.eps, k);
    float ymax = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      h[i] = h[i] * inv * gam[i];
      ymax = fmaxf(ymax, fabsf(h[i]));  // fmaxf skips NaN; columns >= D are 0 or NaN
    }
    int shift = 0;
    if (p.row_scale) {
      shift = clamp_e8m0(rescale_exponent(__float_as_uint(row_max<WPR>(ymax, sm[turn], slot, part, lane)), p.target));
      if (ok && lane == 0 && part == 0) p.row_scale[r] = pow2_float(shift);
    } else if (p.block_scale) {
      // a block is two lanes' chunks
      const float other = __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(ymax), 0xB1, 0xF, 0xF, true));
      shift = clamp_e8m0(rescale_exponent(__float_as_uint(fmaxf(ymax, other)), p.target));
      if (!(lane & 1) && n < (p.D + 127) / 128 * 128 && r < rows)
        p.block_scale[mx_byte(r, n >> 5, groups)] = (uint8_t)(ok ? shift + 127 : 127);
    }
    if (ok && (FULL || valid > 0)) {
      if (p.pre_out) ln_store_f32(p.pre_out + r * (int64_t)p.D + n, valid, h);
      rms_store_any(p.out_fmt, p.out, r * p.ldo + n, valid, h, shift, sat);
    }
  }
}

// Exponents of the gradient: of the norm's part and of the sum's own gradient
// relative to the result's, and the result's.
struct RmsExps {
  int dn, ds, e;
};
__device__ __forceinline__ RmsExps rms_exps(const RmsParams& p) {
  const int en = pow2_exponent(p.s_dy) - pow2_exponent(p.s_x);
  RmsExps x = {0, 0, en};
  if (p.has_res) {
    const int es = pow2_exponent(p.s_res);
    x.e = max(en, es);
    x.dn = en - x.e;
    x.ds = es - x.e;
  }
  return x;
}

// One element of the gradient, the same in the kernel that measures its largest
// magnitude and in the one that casts it (no contraction). The row's numbers are
// a = 2^dn inv, c and k (h, inv and c are those of the row divided by 2^k).
__device__ __forceinline__ float rms_dx(float h, float dy, float gam, float a, float c) {
#pragma clang fp contract(off)
  return (dy * gam - h * c) * a;
}

// Row pass of the backward: the row's two numbers, then the gradient: its amax
// (the dynamic rescale: the second kernel casts) or its codes (none); dgamma's
// partial sums stay in registers over the rows of a workgroup.
template <int XF, int DYF, int WPR, bool FULL>
__global__ __launch_bounds__(rms_threads(WPR)) void rms_bwd_rows_kernel(RmsParams p) {
#pragma clang fp contract(off)
  constexpr int RPW = rms_rpw(WPR);
  constexpr int WAVES = RPW * WPR;
  constexpr bool RANGE = XF == kF32;
  __shared__ float s2[2][RPW][WPR][2], sr[2][RPW][WPR];
  __shared__ float wmax[WAVES];
  __shared__ float red[RPW > 1 ? 1024 * WPR : 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int slot = wave / WPR, part = wave % WPR;
  const int n = 16 * (lane + 64 * part), valid = FULL ? 16 : p.D - n;  // (may be <= 0)
  const bool res = p.has_res != 0, sat = p.sat != 0, direct = p.mode == 0;
  const RmsExps ex = rms_exps(p);
  const int e_out = clamp_e8m0(ex.e);  // (without a rescale)
  float4* rowstats = (float4*)p.partial;
  const int64_t stride = (int64_t)gridDim.x * RPW;
  uint32_t wx[ln_chunk_words<XF>()], wd[ln_chunk_words<DYF>()], wr[8];
  int64_t r0 = (int64_t)blockIdx.x * RPW;
  auto load = [&](int64_t r) {
    const int v = r < p.R ? valid : 0;
    ln_load_raw<XF>(p.x, r * p.ldx + n, v, wx);
    ln_load_raw<DYF>(p.dy, r * p.lddy + n, v, wd);
    if (res) rms_load_any(p.res_fmt, p.res, r * p.ldr + n, v, wr);
  };
  load(r0 + slot);
  float gam[16], pg[16];
  ln_param16(p.gamma, n, max(valid, 0), 1.0f, gam);
#pragma unroll
  for (int i = 0; i < 16; ++i) pg[i] = 0.0f;
  if (blockIdx.x == 0 && threadIdx.x == 0) stat_open(p.hdr, p.tag, nullptr, nullptr);
  float lmax = 0.0f;
  int turn = 0;
#pragma unroll 1
  for (; r0 < p.R; r0 += stride, turn ^= 1) {
    const int64_t r = r0 + slot;
    float h[16], d[16], q[16];
    rms_decode16<XF>(p.x_fmt, wx, h);
    rms_decode16<DYF>(p.dy_fmt, wd, d);
    if (res) rms_decode_any(p.res_fmt, wr, q);
    load(r + stride);
    int k = 0;
    if constexpr (RANGE) k = rms_range<WPR>(h, sr[turn], slot, part, lane);
    float ch = 0.0f, cg = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      ch = fmaf(h[i], h[i], ch);
      cg = fmaf(d[i] * gam[i], h[i], cg);  // columns >= D are 0
    }
    float s[2] = {wave_sum(ch), wave_sum(cg)};
    row_sum<WPR, 2>(s, s2[turn], slot, part, lane);
    const float inv = rms_inv<RANGE>(s[0], p.D, p.eps, k);  // of h / 2^k, which h holds
    const float c = s[1] / (float)p.D * inv * inv;
    const float a = __builtin_ldexpf(inv, ex.dn - k);
    if (r < p.R) {
      if (!direct && lane == 0 && part == 0) rowstats[r] = make_float4(a, c, (float)k, 0.0f);
      float t[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        t[i] = rms_dx(h[i], d[i], gam[i], a, c);
        if (res) t[i] = t[i] + __builtin_ldexpf(q[i], ex.ds);
        lmax = fmaxf(lmax, fabsf(t[i]));  // fmaxf skips NaN; columns >= D are 0 or NaN
        pg[i] = fmaf(d[i], h[i] * inv, pg[i]);
      }
      if (FULL || valid > 0) {
        if (p.pre_out) ln_store_f32(p.pre_out + r * (int64_t)p.D + n, valid, t);
        if (direct) rms_store_any(p.out_fmt, p.out, r * p.ldo + n, valid, t, e_out - ex.e, sat);
      }
    }
  }
  // dgamma's partial row of this workgroup: its row slots added in order
  if (p.dgamma) {
    if constexpr (RPW > 1) {
#pragma unroll 1
      for (int q = 0; q < RPW - 1; ++q) {
        if (slot == q) {
#pragma unroll
          for (int i = 0; i < 16; ++i) red[n + i] = q ? red[n + i] + pg[i] : pg[i];
        }
        __syncthreads();
      }
    }
    if (slot == RPW - 1 && (FULL || valid > 0)) {
      if constexpr (RPW > 1) {
#pragma unroll
        for (int i = 0; i < 16; ++i) pg[i] = red[n + i] + pg[i];
      }
      ln_store_f32(p.partial + 4 * p.R + (int64_t)blockIdx.x * layernorm_param_stride(p.D) + n, valid, pg);
    }
  }
  lmax = wave_max(lmax);
  if (lane == 0) wmax[wave] = lmax;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int i = 1; i < WAVES; ++i) lmax = fmaxf(lmax, wmax[i]);
    stat_await(p.hdr, p.tag, nullptr, nullptr);
    stat_fold(p.hdr, lmax);
  }
}

// (32 rows a workgroup, as the LayerNorm's apply kernel takes for its parameter sums,
// leave 128 workgroups at 4096 x 2048: 32 us, 14 with 8.)
constexpr int RMS_TILE_ROWS = 8;

// The dynamic rescale's second pass: the gradient again from the rows' numbers,
// cast with the rescale that the statistic gives. RMS_TILE_ROWS rows x 2048 columns
// a workgroup, the rows that the first kernel read last taken first (they are
// still in the last-level cache).
template <int XF, int DYF>
__global__ __launch_bounds__(LN_TILE_THREADS) void rms_bwd_apply_kernel(RmsParams p) {
#pragma clang fp contract(off)
  const RmsExps ex = rms_exps(p);
  const int e_out = clamp_e8m0(ex.e + rescale_exponent(p.hdr[0], p.target));
  const int shift = e_out - ex.e;
  const bool sat = p.sat != 0, res = p.has_res != 0;
  const int n = (int)blockIdx.x * LN_TILE_COLS + 16 * (int)threadIdx.x;
  const int valid = p.D - n;
  const int tile = (int)(gridDim.y - 1 - blockIdx.y);
  const float4* rowstats = (const float4*)p.partial;
  if (valid <= 0) return;
  float gam[16];
  ln_param16(p.gamma, n, valid, 1.0f, gam);
  const int64_t r0 = (int64_t)tile * RMS_TILE_ROWS;
  const int64_t r1 = r0 + RMS_TILE_ROWS < p.R ? r0 + RMS_TILE_ROWS : p.R;
  constexpr int PF = 4;  // rows in flight
  uint32_t rx[PF][ln_chunk_words<XF>()], rd[PF][ln_chunk_words<DYF>()], rr[PF][8];
  auto load = [&](int64_t r, uint32_t (&wx)[ln_chunk_words<XF>()], uint32_t (&wd)[ln_chunk_words<DYF>()], uint32_t (&wr)[8]) {
    ln_load_raw<XF>(p.x, r * p.ldx + n, valid, wx);
    ln_load_raw<DYF>(p.dy, r * p.lddy + n, valid, wd);
    if (res) rms_load_any(p.res_fmt, p.res, r * p.ldr + n, valid, wr);
  };
  ln_static_for<0, PF>([&](auto K) {
    constexpr int k = decltype(K)::value;
    if (r0 + k < r1) load(r0 + k, rx[k], rd[k], rr[k]);
  });
#pragma unroll 1
  for (int64_t rb = r0; rb < r1; rb += PF) {
    ln_static_for<0, PF>([&](auto K) {
      constexpr int k = decltype(K)::value;
      const int64_t r = rb + k;
      if (r < r1) {
        const float4 st = rowstats[r];
        float h[16], d[16], q[16], t[16];
        rms_decode16<XF>(p.x_fmt, rx[k], h);
        rms_decode16<DYF>(p.dy_fmt, rd[k], d);
        if (res) rms_decode_any(p.res_fmt, rr[k], q);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          if constexpr (XF == kF32) h[i] = __builtin_ldexpf(h[i], -(int)st.z);
          t[i] = rms_dx(h[i], d[i], gam[i], st.x, st.y);
          if (res) t[i] = t[i] + __builtin_ldexpf(q[i], ex.ds);
        }
        rms_store_any(p.out_fmt, p.out, r * p.ldo + n, valid, t, shift, sat);
        if (r + PF < r1) load(r + PF, rx[k], rd[k], rr[k]);
      }
    });
  }
}

}  // namespace scalify
