// Losses from hidden states x and the output matrix w: softmax cross entropy and
// distillation from a teacher's top logits, without the R x V logits.
//
//   z_ij = s_x s_w r_i (x_i . w_j) / T, lse_i = log sum_j exp z_ij
//   cross entropy (T = 1): loss_i = lse_i - z_i,y_i, dz_ij = g_i (p_ij - [j = y_i])
//   distillation: q_i the softmax of the teacher's t_i / T over its tokens,
//     loss_i = T^2 sum_k q_k (log q_k - z_k + lse_i), dz_ij = g_i T (p_ij - q_ij)
//   dx_i = s_w sum_j dz_ij w_j, dw_j = s_x sum_i dz_ij r_i x_i, p = exp(z - lse)
//
// Rows that do not count (no label or teacher, an upstream gradient of 0) need no
// work: the others are gathered first, as F16, and every product runs over them
// alone. The forward's product (loss_gemm.h) leaves a maximum and a sum for each 128
// columns of a row, which a kernel here joins. The backward goes over w in pieces:
// a piece's logits again, their gradient dz in F16 (rounded once, by up to half a step:
// 2^-11 of a value), dx += dz w and the piece's rows of dw = dz^T x. A piece is as large as 512 MiB of dz
// allow: each one adds to dx, which costs 8 bytes an element and piece.
#include "attention_dev.h"
#include "kernels.h"
#include "loss_dev.h"

#include <algorithm>
#include <type_traits>

namespace scalify {

// ---- which rows count

__device__ __forceinline__ float load_any(const void* base, int fmt, int64_t e) {
  if (fmt == kF32) return ((const float*)base)[e];
  if (fmt == kF16) return decode_hw<kF16>(((const uint16_t*)base)[e]);
  const uint32_t c = ((const uint8_t*)base)[e];
  return fmt == kE4M3 ? decode_hw<kE4M3>(c) : decode_hw<kE5M2>(c);
}
__device__ __forceinline__ float scale_of(const float* s) { return s ? *s : 1.0f; }
__device__ __forceinline__ float wave_sum(float v) {
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// A row's teacher in a wave: entry lane + 64 j in registers j; token -1 where there is none.
constexpr int kTopRegs = kLossMaxTop / 64;
struct TeacherRow {
  int token[kTopRegs];
  float t[kTopRegs];  // logit / T, -Inf where there is no token
};
__device__ __forceinline__ TeacherRow load_teacher(const LossParams& p, int64_t row, int lane) {
  TeacherRow r;
  const float f = scale_of(p.s_t) / p.temp;
#pragma unroll
  for (int j = 0; j < kTopRegs; ++j) {
    const int e = lane + 64 * j;
    r.token[j] = -1;
    r.t[j] = -__builtin_inff();
    if (e < p.top) {
      const int64_t i = p.index[row * p.top + e];
      if (i >= 0 && i < p.V) {
        r.token[j] = (int)i;
        r.t[j] = load_any(p.teacher, p.t_fmt, row * p.ldt + e) * f;
      }
    }
  }
  return r;
}
// Whether a token of the row has a logit above -Inf (a NaN is one).
__device__ __forceinline__ bool teaches(const TeacherRow& r) {
  bool any = false;
#pragma unroll
  for (int j = 0; j < kTopRegs; ++j) any |= r.t[j] != -__builtin_inff();
  return __ballot(any) != 0;
}
// The entries' probabilities, and the logarithms of these.
__device__ __forceinline__ void teacher_softmax(const TeacherRow& r, float (&q)[kTopRegs], float (&logq)[kTopRegs]) {
  float m = -__builtin_inff(), n = 0.f;
#pragma unroll
  for (int j = 0; j < kTopRegs; ++j) m = fmaxf(m, r.t[j]);
  m = wave_max(m);
  if (m == -__builtin_inff()) m = 0.f;
#pragma unroll
  for (int j = 0; j < kTopRegs; ++j) {
    q[j] = expf(r.t[j] - m);
    n += q[j];
  }
  n = wave_sum(n);
  const float l = logf(n);
#pragma unroll
  for (int j = 0; j < kTopRegs; ++j) {
    logq[j] = r.t[j] - m - l;
    q[j] /= n;
  }
}

// Distillation: whether a row has a token of the teacher with a logit above -Inf. A wave a row.
__global__ __launch_bounds__(256) void loss_flags_kernel(LossParams p) {
  const int lane = threadIdx.x & 63;
  for (int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); row < p.R; row += (int64_t)gridDim.x * 4) {
    const TeacherRow r = load_teacher(p, row, lane);
    const bool some = teaches(r);
    if (lane == 0) p.top_on[row] = some;
  }
}

// Rows that count, in order, their number, and the largest upstream gradient and weight in
// dw among them. One workgroup of 16 waves, each with consecutive rows, 64 at a time:
// a first pass counts, a second one places them. Bound: the latency of a wave's chain of
// loads (5 us for 300 rows, 24 for 16384: under 1 % of a call with 32000 tokens of 4096
// columns, 7 % of the backward with 4096 of 512; grids of more workgroups would have to meet in
// between).
__global__ __launch_bounds__(1024) void loss_scan_kernel(LossParams p) {
  __shared__ int sums[16];
  __shared__ float cs[16];
  __shared__ int ws[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t per = (p.R + 1023) / 1024 * 64, lo = wave * per, hi = lo + per < p.R ? lo + per : p.R;
  // (rows' numbers are loaded whether or not they count, four groups at a time)
  int n = 0, most = 0;
  float c = 0.f;
  for (int64_t at = lo; at < hi; at += 256) {
    bool on[4];
    float g[4], r[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t i = at + 64 * j + lane;
      const bool in = i < hi;
      const int64_t label = p.labels && in ? p.labels[i] : -1;
      const int flag = !p.labels && in ? p.top_on[i] : 0;
      g[j] = p.dloss && in ? p.dloss[i] : 1.0f;
      r[j] = p.row_scale && in ? p.row_scale[i] : 1.0f;
      on[j] = (p.labels ? label >= 0 && label < p.V : flag != 0) && g[j] != 0.0f;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint64_t mask = __ballot(on[j]);
      n += (int)__popcll(mask);
      // what a row is, for the second pass: 0 counts
      const int64_t i = at + 64 * j + lane;
      if (i < hi) p.pos[i] = on[j] ? 0 : -1;
      if (on[j]) {
        const float a = fabsf(g[j] * p.temp);
        if (a < __builtin_inff()) c = fmaxf(c, a);
        most = max(most, row_weight(g[j] * p.temp, r[j]));
      }
    }
  }
  c = wave_max(c), most = wave_max(most);
  if (lane == 0) sums[wave] = n, cs[wave] = c, ws[wave] = most;
  __syncthreads();
  int place = 0, all = 0;
  for (int w = 0; w < 16; ++w) {
    if (w < wave) place += sums[w];
    all += sums[w];
  }
  for (int64_t at = lo; at < hi; at += 256) {
    int flag[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t i = at + 64 * j + lane;
      flag[j] = i < hi ? p.pos[i] : -1;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t i = at + 64 * j + lane;
      const uint64_t mask = __ballot(flag[j] >= 0);
      const int to = place + (int)__popcll(mask & (((uint64_t)1 << lane) - 1));
      if (flag[j] >= 0) {
        p.pos[i] = to;
        p.rows[to] = (int)i;
      }
      place += (int)__popcll(mask);
    }
  }
  if (tid == 0) {
    for (int w = 1; w < 16; ++w) c = fmaxf(c, cs[w]), most = max(most, ws[w]);
    p.hdr[LOSS_COUNT] = (uint32_t)all;
    p.hdr[LOSS_CMAX] = __float_as_uint(c);
    p.hdr[LOSS_WEIGHT] = (uint32_t)most;
    p.hdr[LOSS_AMAX_DX] = p.hdr[LOSS_AMAX_DW] = 0u;
  }
}

// Eight codes from element e of a row on, as F16, those past the row's D columns 0.
__device__ __forceinline__ u4 load_tail8(int fmt, const void* base, int64_t e, int left) {
  u4 v = load_f16x8(fmt, base, e);
  if (left < 8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (2 * i >= left) v[i] = 0u;
      else if (2 * i + 1 >= left) v[i] &= 0xFFFFu;
    }
  }
  return v;
}

// A row that counts at its place: x in F16 (D rounded up to 8 columns), and its numbers. ec:
// exponent of the largest upstream gradient; most: the largest row_weight. A workgroup.
__device__ __forceinline__ void gather_row(const LossParams& p, int64_t i, int64_t row, int ec, int most) {
  const int chunks = (p.D + 7) / 8;
  const float g = p.dloss ? p.dloss[row] * p.temp : p.temp;
  const RowUnit unit = row_unit(g, p.row_scale ? p.row_scale[row] : 1.0f, most, ec);
  if (threadIdx.x == 0) {
    p.factor[i] = logit_factor(p, row);
    if (p.labels) p.label[i] = (int)p.labels[row];
    if (p.lse2) {
      p.lse2[i] = p.lse[row] * kLog2e;
      p.coef[i] = ldexpf(g, kLossGradLog2 - unit.dz);
      p.dx_factor[i] = ldexpf(1.0f, unit.dz - ec);
    }
  }
  const float rf = ldexpf(1.0f, unit.x);
  for (int c = threadIdx.x; c < chunks; c += 256) {
    const u4 v = load_tail8(p.x_fmt, p.x, row * p.ldx + 8 * c, p.D - 8 * c);
    *(u4*)((uint16_t*)p.xc + i * p.ldxc + 8 * c) = v;
    if (p.xw) {
      h8 h = __builtin_bit_cast(h8, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) h[k] = (_Float16)((float)h[k] * rf);
      *(h8*)((uint16_t*)p.xw + i * p.ldxc + 8 * c) = h;
    }
  }
}
// Bound: the bytes (16384 x 4096, 8 bits to F16: 201 MB in 51 us).
__global__ __launch_bounds__(256) void loss_gather_kernel(LossParams p) {
  const int count = (int)p.hdr[LOSS_COUNT];
  const int ec = hdr_exponent(p.hdr, LOSS_CMAX), most = (int)p.hdr[LOSS_WEIGHT];
  for (int64_t i = blockIdx.x; i < count; i += gridDim.x) gather_row(p, i, p.rows[i], ec, most);
}

// loss_scan_kernel and loss_gather_kernel in one for at most 128 rows, which every workgroup
// (a row's) scans for itself: 5 us, where two launches took 9. The first one keeps what the
// scan found.
__global__ __launch_bounds__(256) void loss_few_gather_kernel(LossParams p) {
  __shared__ int rows[kLossFewRows], sums[2], ws[2];
  __shared__ float cs[2];
  const int i = threadIdx.x, lane = i & 63, wave = i >> 6;
  static_assert(kLossFewRows == 128, "two waves scan");
  bool on = false;
  uint64_t mask = 0;
  if (i < 128) {
    const bool in = i < p.R;
    const int64_t label = p.labels && in ? p.labels[i] : -1;
    const float g = p.dloss && in ? p.dloss[i] : 1.0f, r = p.row_scale && in ? p.row_scale[i] : 1.0f;
    on = (p.labels ? label >= 0 && label < p.V : in && p.top_on[i] != 0) && g != 0.0f;
    mask = __ballot(on);
    const float a = fabsf(g * p.temp);
    const float c = wave_max(on && a < __builtin_inff() ? a : 0.f);
    const int most = wave_max(on ? row_weight(g * p.temp, r) : 0);
    if (lane == 0) sums[wave] = (int)__popcll(mask), cs[wave] = c, ws[wave] = most;
  }
  __syncthreads();
  const int count = sums[0] + sums[1];
  const float c = fmaxf(cs[0], cs[1]);
  const int most = max(ws[0], ws[1]);
  if (i < 128) {
    const int to = (wave ? sums[0] : 0) + (int)__popcll(mask & (((uint64_t)1 << lane) - 1));
    if (on) rows[to] = i;
    if (blockIdx.x == 0 && i < p.R) {
      p.pos[i] = on ? to : -1;
      if (on) p.rows[to] = i;
    }
  }
  if (blockIdx.x == 0 && i == 0) {
    p.hdr[LOSS_COUNT] = (uint32_t)count;
    p.hdr[LOSS_CMAX] = __float_as_uint(c);
    p.hdr[LOSS_WEIGHT] = (uint32_t)most;
    p.hdr[LOSS_AMAX_DX] = p.hdr[LOSS_AMAX_DW] = 0u;
  }
  __syncthreads();
  if ((int)blockIdx.x < count)
    gather_row(p, blockIdx.x, rows[blockIdx.x], c > 0.f ? floor_log2_bits(__float_as_uint(c)) : 0, most);
}

// n rows of w from v0 on as F16, D rounded up to 8 columns: where 8-bit rows, or those of F16,
// end inside 16 bytes, which the products' loads cannot mask. Bound: the bytes.
__global__ __launch_bounds__(256) void loss_copy_w_kernel(LossParams p, int v0, int n) {
  const int chunks = (p.D + 15) / 16, cols = (p.D + 7) & ~7;
  const int64_t all = (int64_t)n * chunks;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / chunks;
    const int c = 16 * (int)(i - r * chunks);
    uint16_t* o = (uint16_t*)p.w16 + r * p.ldw16 + c;
    const int64_t e = (v0 + r) * p.ldw + c;
    u4 lo, hi;
    if (p.w_fmt == kF16) {
      lo = load_tail8(kF16, p.w, e, p.D - c);
      hi = c + 8 < cols ? load_tail8(kF16, p.w, e + 8, p.D - c - 8) : u4{0u, 0u, 0u, 0u};
    } else {  // (rows of 8 bits hold whole groups of 16)
      const u4 v = *(const u4*)((const uint8_t*)p.w + e);
      lo = to_f16x8(p.w_fmt, u4{v[0], v[1], 0u, 0u});
      hi = to_f16x8(p.w_fmt, u4{v[2], v[3], 0u, 0u});
      if (c + 16 > p.D) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          lo[k] &= (c + 2 * k < p.D ? 0xFFFFu : 0u) | (c + 2 * k + 1 < p.D ? 0xFFFF0000u : 0u);
          hi[k] &= (c + 8 + 2 * k < p.D ? 0xFFFFu : 0u) | (c + 9 + 2 * k < p.D ? 0xFFFF0000u : 0u);
        }
      }
    }
    *(u4*)o = lo;
    if (c + 8 < cols) *(u4*)(o + 8) = hi;
  }
}

// Distillation's forward: the entries of the teacher whose tokens lie in the piece of n rows
// of w from v0 on, of 16 places (a workgroup), by groups of 128 tokens: the product's
// epilogue has such rows and columns at hand. (Which of a group's entries comes first
// changes nothing.) A piece has at most 2^20 tokens. 7 us for 4096 rows of 64 entries; each tile
// searching its rows' lists instead cost the product 38.
constexpr int kMaxBins = (1 << 20) / 128;
__global__ __launch_bounds__(256) void loss_bin_kernel(LossParams p, int v0, int n) {
  __shared__ int at[kMaxBins];
  __shared__ int sums[4];
  const int count = (int)p.hdr[LOSS_COUNT], bins = p.bin_columns, tid = threadIdx.x;
  const int per = (bins + 255) / 256, lo = min(tid * per, bins), hi = min(lo + per, bins);
  for (int64_t g = blockIdx.x; 16 * g < count; g += gridDim.x) {
    for (int i = tid; i < bins; i += 256) at[i] = 0;
    __syncthreads();
    const int all = (int)min((int64_t)16, count - 16 * g) * p.top;
    auto token = [&](int e) {
      const int64_t t = p.index[(int64_t)p.rows[16 * g + e / p.top] * p.top + e % p.top] - v0;
      return t >= 0 && t < n ? (int)t : -1;
    };
    for (int e = tid; e < all; e += 256) {
      const int t = token(e);
      if (t >= 0) atomicAdd(at + t / 128, 1);
    }
    __syncthreads();
    int mine = 0;
    for (int i = lo; i < hi; ++i) mine += at[i];
    int before = mine;
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(before, o, 64);
      if ((tid & 63) >= o) before += v;
    }
    if ((tid & 63) == 63) sums[tid >> 6] = before;
    __syncthreads();
    before -= mine;
    for (int w = 0; w < tid >> 6; ++w) before += sums[w];
    int* const bin = p.bins + g * (bins + 1);
    for (int i = lo; i < hi; ++i) {
      const int k = at[i];
      at[i] = bin[i] = before;
      before += k;
    }
    if (tid == 255) bin[bins] = before;
    __syncthreads();
    for (int e = tid; e < all; e += 256) {
      const int t = token(e);
      if (t >= 0) p.entries[g * 16 * p.top + atomicAdd(at + t / 128, 1)] = bin_pack(e / p.top, t % 128, e % p.top);
    }
    __syncthreads();
  }
}

// Joins the maxima and sums of a row's column groups: log-sum-exp, and the cross
// entropy. 64 places a workgroup, the groups dealt to its 16 waves (a fixed order).
// Rows that do not count get 0. Bound: the bytes, 8 for each row and 128 tokens (16384 rows,
// 32000 tokens: 33 MB in 10 us).
__global__ __launch_bounds__(1024) void loss_join_kernel(LossParams p, int groups) {
  __shared__ float sm[16][64], ss[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int count = (int)p.hdr[LOSS_COUNT];
  for (int64_t b = blockIdx.x; b * 64 < p.R; b += gridDim.x) {
    const int64_t i = b * 64 + lane;
    float m = -__builtin_inff(), n = 0.f;
    if (i < count) {
#pragma unroll 4
      for (int g = wave; g < groups; g += 16) {
        const float2 v = p.stats[(int64_t)g * p.R + i];
        join_sums(m, n, v.x, v.y);
      }
    }
    sm[wave][lane] = m;
    ss[wave][lane] = n;
    __syncthreads();
    if (wave == 0) {
      if (i < count) {
        for (int w = 1; w < 16; ++w) join_sums(m, n, sm[w][lane], ss[w][lane]);
        const float l2 = m + log2f(n);
        const int row = p.rows[i];
        if (p.lse) p.lse[row] = kLn2 * l2;
        if (p.labels) p.loss[row] = kLn2 * (l2 - p.picked2[i]);
      }
      if (p.labels && i < p.R && p.pos[i] < 0) {
        p.loss[i] = 0.f;
        if (p.lse) p.lse[i] = 0.f;
      }
    }
    __syncthreads();
  }
}

// Distillation's loss of a row, from its log-sum-exp l; rows that do not count, and logits of
// tokens that are not there, get 0. A wave.
__device__ __forceinline__ void top_row(const LossParams& p, int64_t row, const TeacherRow& r, float l, int lane) {
  const bool on = teaches(r);
  float q[kTopRegs], logq[kTopRegs], sum = 0.f;
  teacher_softmax(r, q, logq);
#pragma unroll
  for (int j = 0; j < kTopRegs; ++j) {
    const int e = lane + 64 * j;
    if (e >= p.top) continue;
    float* z = p.picked + row * p.top + e;
    if (!on || r.token[j] < 0)
      *z = 0.f;
    else if (q[j] != 0.f)
      sum += q[j] * (logq[j] - (*z - l));
  }
  sum = wave_sum(sum);
  if (lane == 0) {
    p.loss[row] = on ? p.temp * p.temp * sum : 0.f;
    p.lse[row] = on ? l : 0.f;
  }
}
// A wave a row (5 us for 4096 rows of 64 entries).
__global__ __launch_bounds__(256) void loss_top_kernel(LossParams p) {
  const int lane = threadIdx.x & 63;
  for (int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); row < p.R; row += (int64_t)gridDim.x * 4)
    top_row(p, row, load_teacher(p, row, lane), p.lse[row], lane);
}

// The few rows' end: a row's parts joined to its log-sum-exp, and its loss; rows that do not
// count get 0. A workgroup a row. Bound: latency (4 us; the distillation's part in a launch of
// its own took 4 more).
__global__ __launch_bounds__(256) void loss_few_join_kernel(LossParams p, int groups) {
  __shared__ float sm[4], ss[4];
  const int row = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  TeacherRow r;
  if (!p.labels && wave == 0) r = load_teacher(p, row, lane);
  float m = -__builtin_inff(), n = 0.f;
  for (int g = threadIdx.x; g < groups; g += 256) {
    const float2 v = p.stats[(int64_t)row * groups + g];
    join_sums(m, n, v.x, v.y);
  }
  for (int o = 1; o < 64; o <<= 1) join_sums(m, n, __shfl_xor(m, o, 64), __shfl_xor(n, o, 64));
  if (lane == 0) sm[wave] = m, ss[wave] = n;
  __syncthreads();
  if (wave != 0) return;
  m = sm[0], n = ss[0];  // (one value in all lanes)
  for (int w = 1; w < 4; ++w) join_sums(m, n, sm[w], ss[w]);
  const float l2 = m + log2f(n);
  if (!p.labels) {
    top_row(p, row, r, kLn2 * l2, lane);
  } else if (lane == 0) {
    const bool on = p.labels[row] >= 0 && p.labels[row] < p.V;
    p.loss[row] = on ? kLn2 * (l2 - p.picked2[row]) : 0.f;
    if (p.lse) p.lse[row] = on ? kLn2 * l2 : 0.f;
  }
}

// Distillation's backward: dz of the teacher's tokens in the piece of n rows of w from
// v0 on, from their stored logits: c (p - q), q the sum over a token's entries. A wave
// a place. Bound: 2 bytes of every entry's own cache line of dz (8192 rows of 128 entries:
// 48 us, 1 % of the call).
__global__ __launch_bounds__(256) void loss_fix_kernel(LossParams p, int v0, int n) {
  const int lane = threadIdx.x & 63;
  const int count = (int)p.hdr[LOSS_COUNT];
  for (int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); i < count; i += (int64_t)gridDim.x * 4) {
    const int64_t row = p.rows[i];
    const TeacherRow r = load_teacher(p, row, lane);
    float q[kTopRegs], logq[kTopRegs], want[kTopRegs];
    teacher_softmax(r, q, logq);
#pragma unroll
    for (int j = 0; j < kTopRegs; ++j) want[j] = 0.f;
#pragma unroll
    for (int k = 0; k < kTopRegs; ++k)
      for (int o = 0; o < 64 && o + 64 * k < p.top; ++o) {
        const int token = __shfl(r.token[k], o, 64);
        const float add = __shfl(q[k], o, 64);
#pragma unroll
        for (int j = 0; j < kTopRegs; ++j)
          if (r.token[j] == token) want[j] += add;
      }
    const float l2 = p.lse2[i], c = p.coef[i];
#pragma unroll
    for (int j = 0; j < kTopRegs; ++j) {
      const int e = lane + 64 * j, d = r.token[j] - v0;
      if (e < p.top && r.token[j] >= 0 && d >= 0 && d < n) {
        const float prob = exp2f(held_log(p.picked[row * p.top + e] * kLog2e - l2, l2));
        ((_Float16*)p.dz)[i * p.ldz + d] = (_Float16)(c * (prob - want[j]));
      }
    }
  }
}

// ---- the gradients' rescale and cast

// The splits' sum into the first of them, and its statistic (one split's is the product's
// own), of dx or dw. A workgroup a row at a time, or with few rows 1024 columns of it. Bound: the
// bytes (4096 x 2048, two parts: 100 MB in 27 us).
__global__ __launch_bounds__(256) void loss_sum_kernel(LossParams p, int is_dw) {
  const bool dw = is_dw != 0;
  const int count = dw ? p.V : (int)p.hdr[LOSS_COUNT], splits = dw ? p.dw_splits : p.splits;
  const int64_t stride = (int64_t)(dw ? p.V : p.R) * p.ldp;
  float a = 0.f;
  for (int64_t r = blockIdx.x; r < count; r += gridDim.x)
    for (int c = 4 * (int)(blockIdx.y * 256 + threadIdx.x); c < p.D; c += 1024 * gridDim.y) {
      float* o = (dw ? p.dw32 : p.part) + r * p.ldp + c;
      float4 v = *(const float4*)o;
#pragma unroll 4
      for (int s = 1; s < splits; ++s) {
        const float4 w = *(const float4*)(o + s * stride);
        v.x += w.x, v.y += w.y, v.z += w.z, v.w += w.w;
      }
      *(float4*)o = v;
      a = fmaxf(a, fabsf(v.x));
      if (c + 1 < p.D) a = fmaxf(a, fabsf(v.y));
      if (c + 2 < p.D) a = fmaxf(a, fabsf(v.z));
      if (c + 3 < p.D) a = fmaxf(a, fabsf(v.w));
    }
  __shared__ float red[4];
  a = wave_max(a);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = a;
  __syncthreads();
  a = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  if (threadIdx.x == 0) raise_amax(p.hdr + (dw ? LOSS_AMAX_DW : LOSS_AMAX_DX), a);
}

// The gradients' scales and statistics.
__device__ __forceinline__ void write_scale(const LossParams& p, bool dw) {
  if (!(dw ? p.dw_scale : p.dx_scale)) return;
  const int unit = unit_of(p, dw), base = base_of(p, dw);
  *(dw ? p.dw_scale : p.dx_scale) = pow2_float(out_exponent(p, dw, base, unit));
  if (p.amax_out) p.amax_out[dw ? 1 : 0] = ldexpf(__uint_as_float(p.hdr[dw ? LOSS_AMAX_DW : LOSS_AMAX_DX]), unit);
}
__global__ void loss_scales_kernel(LossParams p) { write_scale(p, threadIdx.x == 1); }

// Rows of fp32 products (the sum of `splits` of them) cast to codes; the first cast of
// a call writes the scales too where they are known by then; dx: rows that do not count are 0.
// SUM: there are splits to add. Bound: the bytes (4.7 TB/s for 32000 x 4096 to F16).
template <bool SUM>
__global__ __launch_bounds__(256) void loss_cast_kernel(LossParams p, int is_dw, int scales, int splits) {
  const bool dw = is_dw != 0;
  if (scales && blockIdx.x == 0 && threadIdx.x < 2) write_scale(p, threadIdx.x == 1);
  const int unit = unit_of(p, dw), base = base_of(p, dw), e_out = out_exponent(p, dw, base, unit);
  const int shift = e_out - base - unit, chunks = (p.D + 15) / 16;
  const int64_t all = (int64_t)(dw ? p.V : p.R) * chunks;
  const float* src = dw ? p.dw32 : p.part;
  void* out = dw ? p.dw : p.dx;
  const int fmt = dw ? p.dw_fmt : p.dx_fmt;
  const int64_t ldo = dw ? p.lddw : p.lddx;
  const int64_t stride = (int64_t)(dw ? p.V : p.R) * p.ldp;
  const bool stat = SUM && p.mode != 1 && p.amax_out;  // (one product's is its own kernel's)
  float lmax = 0.f;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / chunks;
    const int c = 16 * (int)(i - r * chunks), cols = p.D - c;
    const int64_t from = dw ? r : p.pos[r];
    uint32_t u[16];
    if (dw && fmt != kF16 && p.dw_splits == 1) {
      load16<kF16>(src, from * p.ldp + c, u);  // (16 bits of each fp32, sticky16)
#pragma unroll
      for (int k = 0; k < 16; ++k) u[k] <<= 16;
    } else if (from >= 0) {
      load16<kF32>(src, from * p.ldp + c, u);
#pragma unroll 4
      for (int k = 1; k < (SUM ? splits : 1); ++k) {
        uint32_t w[16];
        load16<kF32>(src, k * stride + from * p.ldp + c, w);
#pragma unroll
        for (int j = 0; j < 16; ++j) u[j] = __float_as_uint(__uint_as_float(u[j]) + __uint_as_float(w[j]));
      }
      if (stat) {
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (j < cols) lmax = fmaxf(lmax, fabsf(__uint_as_float(u[j])));
      }
    } else {
#pragma unroll
      for (int k = 0; k < 16; ++k) u[k] = 0u;
    }
    const int64_t e = r * ldo + c;
    if (fmt == kF16) store_codes<kF16>(out, e, u, cols, shift, p.sat);
    else if (fmt == kE4M3) store_codes<kE4M3>(out, e, u, cols, shift, p.sat);
    else store_codes<kE5M2>(out, e, u, cols, shift, p.sat);
  }
  if (stat) {
    lmax = wave_max(lmax);
    if ((threadIdx.x & 63) == 0) raise_amax(p.hdr + (dw ? LOSS_AMAX_DW : LOSS_AMAX_DX), lmax);
  }
}

// The few rows' dx from its many parts: 256 columns of a row a workgroup, whose waves share
// the parts (a thread for 16 columns, as above: 22 us for 16 rows of 2048 columns and 64
// parts, now 5). KEEP: the sums take the place of the first part (the statistic of the dynamic
// rescale is due before its cast); else they are cast at once.
template <bool KEEP>
__global__ __launch_bounds__(256) void loss_few_sum_kernel(LossParams p, int scales) {
  __shared__ __attribute__((aligned(16))) float sums[4][256], most[4];
  const int i = threadIdx.x, lane = i & 63, wave = i >> 6;
  const int col0 = 256 * blockIdx.y, c4 = col0 + 4 * lane, col = col0 + i;
  if (scales && blockIdx.x == 0 && blockIdx.y == 0 && i < 2) write_scale(p, i == 1);
  const int unit = unit_of(p, false), base = base_of(p, false), shift = out_exponent(p, false, base, unit) - base - unit;
  float lmax = 0.f;
  for (int64_t row = blockIdx.x; row < p.R; row += gridDim.x) {
    const int64_t from = p.pos[row];
    if (KEEP && from < 0) continue;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (from >= 0 && c4 < p.D) {
      const float* o = p.part + from * p.ldp + c4;
#pragma unroll 8
      for (int s = wave; s < p.splits; s += 4) {
        const float4 w = *(const float4*)(o + (int64_t)s * p.R * p.ldp);
        v.x += w.x, v.y += w.y, v.z += w.z, v.w += w.w;
      }
    }
    __syncthreads();
    *(float4*)&sums[wave][4 * lane] = v;
    __syncthreads();
    const float t = (sums[0][i] + sums[1][i]) + (sums[2][i] + sums[3][i]);
    if (col < p.D) lmax = fmaxf(lmax, fabsf(t));
    if constexpr (KEEP) {
      if (col < p.D) p.part[from * p.ldp + col] = t;
    } else {
      sums[0][i] = t;  // (its own column's alone)
      __syncthreads();
      const int c = col0 + 16 * i, cols = p.D - c;
      if (i < 16 && cols > 0) {
        uint32_t u[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) u[k] = __float_as_uint(sums[0][16 * i + k]);
        const int64_t e = row * p.lddx + c;
        if (p.dx_fmt == kF16) store_codes<kF16>(p.dx, e, u, cols, shift, p.sat);
        else if (p.dx_fmt == kE4M3) store_codes<kE4M3>(p.dx, e, u, cols, shift, p.sat);
        else store_codes<kE5M2>(p.dx, e, u, cols, shift, p.sat);
      }
    }
  }
  if (KEEP || p.amax_out) {
    lmax = wave_max(lmax);
    if (lane == 0) most[wave] = lmax;
    __syncthreads();
    if (i == 0) raise_amax(p.hdr + LOSS_AMAX_DX, fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])));
  }
}

// ---- host

static int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

LossPlan loss_plan(int64_t R, int64_t V, int64_t D, int w_fmt, int top, bool back, bool amax, LossParams* p, void* base) {
  LossPlan z = {};
  // w is copied as F16 where its rows end inside a group of 16 bytes
  z.copy_w = D % (w_fmt == kF16 ? 8 : 16) != 0;
  // (a pitch of an odd number of 128 bytes: rows of a power of two would share memory channels)
  auto pitch = [](int64_t cols) { return up(cols, 64) + (up(cols, 64) / 64 % 2 == 0 ? 64 : 0); };
  z.ldxc = z.ldw16 = pitch(D);
  z.ldp = up(D, 16);
  // rows of w at a time: 512 MiB of dz, 512 MiB of decoded w
  int64_t most = (int64_t)1 << 20;
  if (back && R > 0) most = std::min(most, std::max<int64_t>(256, ((int64_t)1 << 28) / R / 256 * 256));
  if (z.copy_w) most = std::min(most, std::max<int64_t>(256, ((int64_t)1 << 28) / z.ldw16 / 256 * 256));
  if (back && loss_few_bwd(R, V)) most = V;
  const int64_t pieces = (V + most - 1) / most;
  z.piece = (int)up((V + pieces - 1) / pieces, 256);
  z.ldz = pitch(z.piece);
  z.splits = z.dw_splits = 1;
  if (back) {
    // dx has few tiles: its k is split where that fills the device's rounds of tiles (4.9e12
    // operations a second and CU) for more than the sums' bytes cost (4e12 a second)
    const int64_t cus = gemm4_grid(1 << 30), columns = (D + 255) / 256;
    auto best_of = [&](int64_t rows, int64_t k, auto bytes) {
      double best = 1e300;
      int splits = 1;
      for (int s = 1; s <= 64 && (s == 1 || k / s >= 256); ++s) {
        const int64_t tiles = (rows + 255) / 256 * columns * s;
        const double t = (double)((tiles + cus - 1) / cus) / s * 2.0 * 65536.0 * (double)k / 4.9e12 + bytes(s) / 4e12;
        if (t < best * 0.98) best = t, splits = s;
      }
      return splits;
    };
    z.splits = best_of(R, z.piece, [&](int s) { return 8.0 * s * (double)R * (double)D; });
    // dw likewise over the rows, where V and D are small (one part leaves as codes, or as its own
    // fp32; 16384 rows, 4096 x 512: 326 us, was 532)
    z.dw_splits = best_of(std::min<int64_t>(z.piece, V), R, [&](int s) { return s == 1 ? 0.0 : (8.0 * s + 8.0) * (double)V * (double)D; });
  }
  const bool few = back ? loss_few_bwd(R, V) : R <= kLossFewRows;
  if (back && few) {
    // a workgroup 128 columns of dx and a part of the vocabulary: 4 for each CU, 2 where the
    // parts' sums are more bytes
    const int64_t tiles = (D + 127) / 128, most = (V + 63) / 64, per_cu = R <= 32 ? 4 : 2;
    z.splits = (int)std::min(std::min<int64_t>(256, most), std::max<int64_t>(1, per_cu * gemm4_grid(1 << 30) / tiles));
  }
  size_t at = kHeaderBytes;
  auto take = [&](auto** to, size_t bytes) {
    if (p) *to = (std::remove_reference_t<decltype(**to)>*)((uint8_t*)base + at);
    at += (bytes + 255) / 256 * 256;
  };
  LossParams none;
  LossParams& q = p ? *p : none;
  if (p) p->hdr = (uint32_t*)base;
  const size_t r = (size_t)R;
  take(&q.rows, 4 * r);
  take(&q.pos, 4 * r);
  take(&q.factor, 4 * r);
  take(&q.label, 4 * r);
  if (top) take(&q.top_on, 4 * r);
  auto bytes_of = [](int64_t rows, int64_t ld, int64_t size) { return (size_t)rows * (size_t)ld * (size_t)size; };
  uint16_t *xc = nullptr, *xw = nullptr, *w16 = nullptr, *dz = nullptr;
  if (back || !few) take(&xc, bytes_of(R, z.ldxc, 2));
  if (z.copy_w && !few) take(&w16, bytes_of(std::min<int64_t>(z.piece, V), z.ldw16, 2));
  if (back) {
    take(&q.lse2, 4 * r);
    take(&q.coef, 4 * r);
    take(&q.dx_factor, 4 * r);
    take(&xw, bytes_of(R, z.ldxc, 2));
    take(&dz, bytes_of(R, z.ldz, 2));
    take(&q.part, bytes_of(R, z.ldp, 4 * (int64_t)z.splits));
    if ((amax || z.dw_splits > 1) && !few) take(&q.dw32, bytes_of(V, z.ldp, 4 * (int64_t)z.dw_splits));
  } else {
    if (top) {
      float *lse = nullptr, *picked = nullptr;
      take(&lse, 4 * r);
      take(&picked, 4 * r * (size_t)top);
      if (p && !p->lse) p->lse = lse;
      if (p && !p->picked) p->picked = picked;
    }
    if (top && !few) {
      const size_t groups = (size_t)((R + 15) / 16);
      q.bin_columns = (int)((std::min<int64_t>(z.piece, V) + 127) / 128);
      take(&q.bins, 4 * groups * (size_t)(q.bin_columns + 1));
      take(&q.entries, 64 * groups * (size_t)top);
    }
    take(&q.picked2, 4 * r);
    take(&q.stats, 8 * r * (size_t)(few ? (V + 63) / 64 : 2 * ((V + 255) / 256)));
  }
  if (p) {
    p->xc = xc;
    p->xw = back && p->dw_scale && (p->row_scale || p->dloss) ? xw : nullptr;  // (else x as it is)
    p->w16 = few ? nullptr : w16;
    p->dz = dz;
    p->ldxc = z.ldxc;
    p->ldw16 = z.ldw16;
    p->ldz = z.ldz;
    p->ldp = z.ldp;
    p->piece = z.piece;
    p->splits = z.splits;
    p->dw_splits = z.dw_splits;
  }
  z.bytes = at;
  return z;
}

static int64_t groups_for(int64_t n, int64_t each, int64_t most) {
  const int64_t g = (n + each - 1) / each;
  return g < 1 ? 1 : (g < most ? g : most);
}

// A workgroup a CU, one at least (no rows: it leaves at once).
static int grid_for(int64_t tiles) { return std::max(1, gemm4_grid((int)tiles)); }

#define TRY(call)                        \
  do {                                   \
    const hipError_t e_ = (call);        \
    if (e_ != hipSuccess) return e_;     \
  } while (0)

// Rows that count and their x.
static hipError_t begin_loss(const LossParams& p, hipStream_t s) {
  if (!p.labels) TRY(launch_one(loss_flags_kernel, groups_for(p.R, 4, 8192), 256, s, p));
  if (p.R > 0 && p.R <= kLossFewRows) return launch_one(loss_few_gather_kernel, p.R, 256, s, p);
  TRY(launch_one(loss_scan_kernel, 1, 1024, s, p));
  return launch_one(loss_gather_kernel, groups_for(p.R, 1, 16384), 256, s, p);
}

// The product of a piece's logits.
static hipError_t piece_logits(const LossParams& p, int v0, int n, int epi, LossGemm* g, hipStream_t s) {
  *g = LossGemm{};
  if (p.w16) TRY(launch_one(loss_copy_w_kernel, groups_for((int64_t)n * ((p.D + 15) / 16), 1024, 16384), 256, s, p, v0, n));
  g->a = p.xc;
  g->lda = 2 * p.ldxc;
  const int64_t pitch = p.ldw * (p.w_fmt == kF16 ? 2 : 1);
  g->b = p.w16 ? p.w16 : (const void*)((const uint8_t*)p.w + (int64_t)v0 * pitch);
  g->ldb = p.w16 ? 2 * p.ldw16 : pitch;
  g->b_fmt = p.w16 ? kF16 : p.w_fmt;
  g->M = p.R;
  g->N = n;
  g->K = p.D;
  g->hdr = p.hdr;
  g->splits = 1;
  g->v0 = v0;
  g->factor = p.factor;
  g->lse2 = p.lse2;
  g->coef = p.coef;
  g->dx_factor = p.dx_factor;
  g->label = p.labels ? p.label : nullptr;
  g->picked2 = p.picked2;
  g->bins = p.bins;
  g->entries = p.entries;
  g->bin_columns = p.bin_columns;
  g->top = p.top;
  g->rows = p.rows;
  g->picked = p.picked;
  g->stats = p.stats;
  g->R = p.R;
  g->dz = p.dz;
  g->ldz = p.ldz;
  const int64_t tiles = (int64_t)((p.R + 255) / 256) * ((n + 255) / 256);
  return launch_loss_logits(*g, epi, grid_for(tiles), s);
}

hipError_t launch_loss_fwd(const LossParams& p, hipStream_t s) {
  if (p.R <= kLossFewRows) {
    TRY(launch_loss_few(p, s));
    return launch_one(loss_few_join_kernel, p.R, 256, s, p, loss_few_groups(p));
  }
  TRY(begin_loss(p, s));
  LossGemm g;
  for (int v0 = 0; v0 < p.V; v0 += p.piece) {
    const int n = std::min(p.piece, p.V - v0);
    if (!p.labels) TRY(launch_one(loss_bin_kernel, groups_for(p.R, 16, 16384), 256, s, p, v0, n));
    TRY(piece_logits(p, v0, n, p.labels ? LOSS_STATS : LOSS_PICK, &g, s));
  }
  TRY(launch_one(loss_join_kernel, groups_for(p.R, 64, 16384), 1024, s, p, 2 * ((p.V + 255) / 256)));
  if (!p.labels) TRY(launch_one(loss_top_kernel, groups_for(p.R, 4, 8192), 256, s, p));
  return hipSuccess;
}

hipError_t launch_loss_bwd(const LossParams& p, hipStream_t s) {
  TRY(begin_loss(p, s));
  const bool few = loss_few_bwd(p.R, p.V), parts_dw = !few && p.dw_splits > 1;
  if (few) {
    TRY(launch_loss_few_dz(p, s));
    if (!p.labels) TRY(launch_one(loss_fix_kernel, groups_for(p.R, 4, 8192), 256, s, p, 0, p.V));
    TRY(launch_loss_few_grads(p, s));
  }
  for (int v0 = few ? p.V : 0; v0 < p.V; v0 += p.piece) {
    const int n = std::min(p.piece, p.V - v0);
    LossGemm g;
    TRY(piece_logits(p, v0, n, LOSS_DZ, &g, s));
    if (!p.labels) TRY(launch_one(loss_fix_kernel, groups_for(p.R, 4, 8192), 256, s, p, v0, n));
    const void* w = g.b;
    const int64_t ldw = g.ldb;
    if (p.dx_scale) {
      g.a = p.dz;
      g.lda = 2 * p.ldz;
      g.b = w;
      g.ldb = ldw;
      g.M = p.R;
      g.N = p.D;
      g.K = n;
      g.splits = p.splits;
      g.part_rows = p.R;
      g.part = p.part;
      g.ldp = p.ldp;
      g.accumulate = v0 > 0;
      g.amax = p.splits == 1 && v0 + n == p.V ? p.hdr + LOSS_AMAX_DX : nullptr;
      const int64_t tiles = (int64_t)((p.R + 255) / 256) * ((p.D + 255) / 256) * p.splits;
      TRY(launch_loss_grads(g, LOSS_DX, grid_for(tiles), s));
    }
    if (p.dw_scale) {
      g.a = p.dz;
      g.lda = 2 * p.ldz;
      g.b = p.xw ? p.xw : p.xc;
      g.ldb = 2 * p.ldxc;
      g.M = n;
      g.N = p.D;
      g.K = 0;
      g.count_is = 1;
      g.splits = p.dw_splits;
      g.part = p.dw32;
      g.part_rows = p.V;
      g.ldp = p.ldp;
      g.out = p.dw;
      g.ldo = p.lddw;
      g.out_fmt = parts_dw ? kF16 : p.dw_fmt;  // (parts: as the dynamic rescale's F16, in fp32)
      g.sat = p.sat;
      g.mode = parts_dw ? 1 : p.mode;
      g.amax = parts_dw ? nullptr : p.hdr + LOSS_AMAX_DW;
      g.s0 = p.s_dloss;
      g.s1 = p.s_x;
      const int64_t tiles = (int64_t)((n + 255) / 256) * ((p.D + 255) / 256) * p.dw_splits;
      TRY(launch_loss_grads(g, LOSS_DW, grid_for(tiles), s));
    }
  }
  // The dynamic rescale needs a statistic before its cast, and so the parts' sum; else the cast
  // sums, and the statistic, if it is asked for, is written behind it.
  const bool amax = p.mode == 1, late = !amax && p.amax_out;
  auto launch2 = [&](auto kernel, int64_t x, unsigned y, auto... args) {
    LossParams q = p;
    void* a[] = {&q, &args...};
    const hipError_t e = hipLaunchKernel((const void*)kernel, dim3((unsigned)x, y), dim3(256), a, 0, s);
    if (e != hipSuccess) (void)hipGetLastError();
    return e;
  };
  // (512 and 1024 workgroups: more of them wait for each other at the statistic's word; 4096 rows
  // of 2048 columns, a workgroup each, took 48 us, now 27)
  auto sum_and_cast = [&](int is_dw, int rows, int splits, int scales) {
    if (amax && splits > 1) TRY(launch2(loss_sum_kernel, groups_for(rows, 1, 1024), rows < 1024 ? (unsigned)groups_for(p.D, 1024, 64) : 1u, is_dw));
    const int parts = amax ? 1 : splits;
    return launch_one(parts > 1 ? loss_cast_kernel<true> : loss_cast_kernel<false>, groups_for((int64_t)rows * ((p.D + 15) / 16), 256, 16384), 256, s, p, is_dw,
                      scales, parts);
  };
  if (p.dx_scale && few) {
    const unsigned wide = (unsigned)((p.D + 255) / 256);
    const int64_t rows = groups_for(p.R, 1, std::max<int64_t>(1, 512 / wide));
    if (amax) {
      TRY(launch2(loss_few_sum_kernel<true>, rows, wide, 0));
      TRY(sum_and_cast(0, p.R, 1, 1));
    } else {
      TRY(launch2(loss_few_sum_kernel<false>, rows, wide, late ? 0 : 1));
    }
  }
  // (the scales need both statistics: dw's parts are summed before the first cast)
  const bool cast_dw = p.dw_scale && !few && (amax || parts_dw);
  if (cast_dw) TRY(sum_and_cast(1, p.V, p.dw_splits, 0));
  if (p.dx_scale && !few) TRY(sum_and_cast(0, p.R, p.splits, late ? 0 : 1));
  const bool written = !late && p.dx_scale;
  return written ? hipSuccess : launch_one(loss_scales_kernel, 1, 2, s, p);
}

}  // namespace scalify
