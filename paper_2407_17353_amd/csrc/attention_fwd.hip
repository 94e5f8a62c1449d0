// Attention forward: softmax(alpha q k^T) v in one pass over the keys with the
// running maximum and sum of every row.
//
// A workgroup holds query columns -- (position, head) pairs of the heads that
// share a key head, so a tile of keys is read once for all of them -- and walks
// tiles of keys. Scores are formed transposed (keys x queries): a lane then owns
// one query, its softmax needs one exchange (with lane ^ 32), and the
// probabilities are the next product's operand as they stand.
//
//   wide (128 columns, 32 a wave; tiles of 64 keys that the waves share):
//     prompts and training; bound by the matrix cores and the exponentials;
//   narrow (32 columns; the waves take a quarter each of a tile of 128 keys and
//     are joined at the end): single tokens; bound by reading the cache.
// Where that leaves the device idle the keys of a sequence are split over
// workgroups, whose unnormalised results a second kernel joins.
#include "attention_dev.h"
#include "kernels.h"

namespace scalify {

template <int DP, bool NARROW>
__global__ __launch_bounds__(256, 2) void attn_fwd_kernel(AttnParams p, int tiles) {
  constexpr int TK = NARROW ? 128 : 64, NB = NARROW ? 1 : 2, KS = DP / 16, DB = DP / 32;
  constexpr int COLS = NARROW ? 32 : 128;
  __shared__ __align__(16) uint8_t lds[2 * TK * DP * 2];
  __shared__ int odd;
  uint8_t* const kt = lds;
  uint8_t* const vt = lds + TK * DP * 2;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), h = lane >> 5;
  const Place at = attn_place(p);
  const int split = (int)(at.rest % p.splits);
  // (the last columns see the most keys where the mask is causal: they go first)
  const int tile = tiles - 1 - (int)(at.rest / p.splits);
  const Seq sq = load_seq(p, at.b);
  const int64_t ncols = (int64_t)sq.lq * p.G;
  const int64_t col0 = (int64_t)tile * COLS;
  if (blockIdx.x == 0 && threadIdx.x == 0) *p.out_scale = pow2_float(clamp_e8m0(pow2_exponent(p.s_v)));
  if (col0 >= ncols) return;

  // This lane's query.
  const int64_t col = col0 + (NARROW ? 0 : 32 * wave) + (lane & 31);
  const bool live = col < ncols;
  const int pos = (int)(col / p.G), head = at.hk * p.G + (int)(col - (int64_t)pos * p.G);
  const int64_t qrow = sq.q0 + pos;
  const int behind = sq.lk - sq.lq;  // causal: query i sees keys up to i + behind
  // (a lane without a query sees every key: its result goes nowhere)
  const int last = !live ? 0x7FFFFFFF : (p.causal ? min(pos + behind, sq.lk - 1) : sq.lk - 1);
  const int last0 = p.causal ? min((int)(col0 / p.G) + behind, sq.lk - 1) : sq.lk - 1;  // of the first column
  h8 qf[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks)
    qf[ks] = row_chunk(p.q_fmt, p.q, qrow * p.ldq + (int64_t)head * p.D, ks, h, p.D, live);
  // Keys of this workgroup: those that its last column sees, this split's share
  // in whole tiles.
  const int64_t last_col = col0 + COLS < ncols ? col0 + COLS - 1 : ncols - 1;
  const int seen = p.causal ? max(0, min(sq.lk, (int)(last_col / p.G) + behind + 1)) : sq.lk;
  const int share = ((seen + p.splits - 1) / p.splits + TK - 1) / TK * TK;
  const int begin = (int)min((int64_t)split * share, (int64_t)seen), end = min(seen, begin + share);

  const float c1 = score_factor(p);
  float m = neg_inf(), l = 0.0f;
  f16v acc[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) acc[d] = f16v{};

  TileLoader<TK, DP, 256> lk, lv;
  lk.init(p.k, sq.k0 * p.ldk + (int64_t)at.hk * p.D, p.ldk, p.D, p.k_fmt);
  lv.init(p.v, sq.k0 * p.ldv + (int64_t)at.hk * p.D, p.ldv, p.D, p.v_fmt);

  auto compute = [&](int key0) {
    float s[NB][16];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      f16v c = {};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        c = mfma(row_operand<DP>(kt, NARROW ? 32 * wave : 32 * b, ks, lane), qf[ks], c);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[b][r] = c[r];
    }
    if (__any(key0 + 32 * NB - 1 > last)) {
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (key0 + 32 * b + result_row(r, h) > last) s[b][r] = neg_inf();
    }
    float top = s[0][0];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, s[b][r]);  // (fmaxf skips NaN)
    top = fmaxf(top, other_half(top, h)) * c1;
    if (__any(top > m)) {
      const float now = fmaxf(m, top);
      const float f = now == neg_inf() ? 1.0f : __builtin_amdgcn_exp2f(m - now);
      m = now;
      l *= f;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[d][r] *= f;
    }
    const float off = kProbLog2 - (m == neg_inf() ? 0.0f : m);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[b][r] = __builtin_amdgcn_exp2f(fmaf(s[b][r], c1, off));
        l += s[b][r];
      }
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const h8 pf = to_operand(s[b], g);
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          const h8 vf = col_operand<DP>(vt, (NARROW ? 32 * wave : 32 * b) + 16 * g, d, lane);
          acc[d] = mfma(vf, pf, acc[d]);
        }
      }
    }
  };
  // Values that are not finite, in a tile that the mask cuts: added pair by pair
  // (an admitted probability is positive, so its product with an infinity is that
  // infinity), and taken out of the tile.
  auto odd_values = [&](int key0) {
#pragma unroll 1
    for (int j = 0; j < 32 * NB; ++j) {
      if (key0 + j > last) continue;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const u2 w = *(const u2*)(vt + tile_off<DP>((NARROW ? 32 * wave : 0) + j, 4 * d + g) + 8 * h);
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[d][4 * g + i] += odd_part((w[i >> 1] >> (16 * (i & 1))) & 0xFFFFu);
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < TK * DP / 8; i += 256)
      ((h8*)vt)[i] = finite_part(((const h8*)vt)[i]);
    __syncthreads();
  };

  if (threadIdx.x == 0) odd = -1;
  __syncthreads();
  if (begin < end) {
    lk.load(begin, end);
    lv.load(begin, end);
  }
#pragma unroll 1
  for (int t = begin; t < end; t += TK) {
    lk.store(kt);
    lv.store(vt);
    if (t + TK - 1 > last0) mark_not_finite(lv, &odd, t);
    __syncthreads();
    if (t + TK < end) {
      lk.load(t + TK, end);
      lv.load(t + TK, end);
    }
    const int key0 = t + (NARROW ? 32 * wave : 0);
    if (__builtin_amdgcn_readfirstlane(odd) == t) odd_values(key0);
    compute(key0);
    __syncthreads();
  }
  l += other_half(l, h);

  auto finish = [&](int d, const f16v& o, float m1, float l1, int64_t c, int hd, int64_t row) {
    // Block d (32 columns) of a query's result: registers 4 g ... are consecutive columns.
    const float inv = l1 == 0.0f ? 0.0f : 1.0f / l1;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int n = 32 * d + 8 * g + 4 * h;
      if (n < p.D) {
        float y[4];
        if (p.splits > 1) {
          *(float4*)(p.part_o + ((split * p.rows_q + row) * p.H + hd) * (int64_t)p.D + n) =
              make_float4(o[4 * g], o[4 * g + 1], o[4 * g + 2], o[4 * g + 3]);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) y[i] = l1 == 0.0f ? 0.0f : o[4 * g + i] * inv;
          store4_any(p.out_fmt, p.out, row * p.ldo + (int64_t)hd * p.D + n, y, 0, p.sat != 0);
        }
      }
    }
  };
  auto finish_row = [&](float m1, float l1, int hd, int64_t row) {
    if (p.splits > 1) p.part_ml[(split * p.rows_q + row) * p.H + hd] = make_float2(m1, l1);
    else if (p.lse)
      p.lse[(int64_t)hd * p.rows_q + row] = l1 == 0.0f ? neg_inf() : (m1 - kProbLog2 + __builtin_amdgcn_logf(l1)) * kLn2;
  };

  if constexpr (!NARROW) {
    if (live) {
#pragma unroll
      for (int d = 0; d < DB; ++d) finish(d, acc[d], m, l, col, head, qrow);
      if (h == 0) finish_row(m, l, head, qrow);
    }
  } else {
    // Join the four waves: maxima and sums first, then the scaled results, of
    // which wave w adds block w.
    float2* ml = (float2*)lds;
    if (h == 0) ml[wave * 32 + lane] = make_float2(m, l);
    __syncthreads();
    float top = neg_inf(), sum = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, ml[w * 32 + (lane & 31)].x);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float2 v = ml[w * 32 + (lane & 31)];
      sum += v.x == neg_inf() ? v.y : v.y * __builtin_amdgcn_exp2f(v.x - top);
    }
    const float f = m == neg_inf() ? 1.0f : __builtin_amdgcn_exp2f(m - top);
    __syncthreads();
    float* part = (float*)lds;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) part[((wave * DB + d) * 16 + r) * 64 + lane] = acc[d][r] * f;
    __syncthreads();
    if (wave < DB && live) {
      f16v o;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float a = part[(wave * 16 + r) * 64 + lane];
#pragma unroll
        for (int w = 1; w < 4; ++w) a += part[((w * DB + wave) * 16 + r) * 64 + lane];
        o[r] = a;
      }
      finish(wave, o, top, sum, col, head, qrow);
      if (wave == 0 && h == 0) finish_row(top, sum, head, qrow);
    }
  }
}

// Joins the splits of a query: 32 lanes, four columns each.
__global__ __launch_bounds__(256) void attn_join_kernel(AttnParams p) {
  const int lane = threadIdx.x & 31;
  const Place at = attn_place(p);
  const Seq sq = load_seq(p, at.b);
  const int64_t col = at.rest * 8 + (threadIdx.x >> 5);
  if (col >= (int64_t)sq.lq * p.G) return;
  const int pos = (int)(col / p.G), head = at.hk * p.G + (int)(col - (int64_t)pos * p.G);
  const int64_t row = sq.q0 + pos;
  float m = neg_inf();
  for (int s = 0; s < p.splits; ++s) m = fmaxf(m, p.part_ml[(s * p.rows_q + row) * p.H + head].x);
  float l = 0.0f, y[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s = 0; s < p.splits; ++s) {
    const int64_t i = (s * p.rows_q + row) * p.H + head;
    const float2 ml = p.part_ml[i];
    if (ml.y == 0.0f) continue;  // (nothing admitted)
    const float f = ml.x == neg_inf() ? 1.0f : __builtin_amdgcn_exp2f(ml.x - m);
    l += ml.y * f;
    if (4 * lane < p.D) {
      const float4 o = *(const float4*)(p.part_o + i * p.D + 4 * lane);
      y[0] += o.x * f;
      y[1] += o.y * f;
      y[2] += o.z * f;
      y[3] += o.w * f;
    }
  }
  if (4 * lane < p.D) {
    const float inv = 1.0f / l;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = l == 0.0f ? 0.0f : y[i] * inv;
    store4_any(p.out_fmt, p.out, row * p.ldo + (int64_t)head * p.D + 4 * lane, y, 0, p.sat != 0);
  }
  if (p.lse && lane == 0)
    p.lse[(int64_t)head * p.rows_q + row] = l == 0.0f ? neg_inf() : (m - kProbLog2 + __builtin_amdgcn_logf(l)) * kLn2;
}

__global__ void attn_scale_kernel(AttnParams p) { *p.out_scale = pow2_float(clamp_e8m0(pow2_exponent(p.s_v))); }

// 512 workgroups (two on each of the 256 CUs) fill the device; a split is worth
// its second kernel from 256 keys on.
AttnPlan attention_plan(int64_t batch, int Hkv, int G, int64_t max_q, int64_t max_k) {
  AttnPlan r;
  const int64_t cols = max_q * G;
  r.narrow = cols <= 32;
  const int64_t groups = batch * Hkv * ((cols + (r.narrow ? 31 : 127)) / (r.narrow ? 32 : 128));
  int64_t s = groups > 0 ? 512 / groups : 1;
  if (s > max_k / 256) s = max_k / 256;
  if (s > 64) s = 64;
  r.splits = s < 2 ? 1 : (int)s;
  return r;
}

template <int DP>
static void launch(const AttnParams& p, const AttnPlan& plan, hipStream_t s) {
  const int64_t cols = p.max_q * p.G;
  const int tiles = (int)((cols + (plan.narrow ? 31 : 127)) / (plan.narrow ? 32 : 128));
  const dim3 g((unsigned)(p.batch * p.Hkv * tiles * plan.splits)), b(256);
  if (plan.narrow) hipLaunchKernelGGL((attn_fwd_kernel<DP, true>), g, b, 0, s, p, tiles);
  else hipLaunchKernelGGL((attn_fwd_kernel<DP, false>), g, b, 0, s, p, tiles);
}

hipError_t launch_attention_fwd(const AttnParams& p, const AttnPlan& plan, hipStream_t s) {
  if (p.rows_q == 0 || p.batch == 0 || p.max_q == 0) {
    hipLaunchKernelGGL(attn_scale_kernel, dim3(1), dim3(1), 0, s, p);
    return hipGetLastError();
  }
  if (p.D <= 64) launch<64>(p, plan, s);
  else launch<128>(p, plan, s);
  if (plan.splits > 1) {
    const int64_t cols = p.max_q * p.G;
    hipLaunchKernelGGL(attn_join_kernel, dim3((unsigned)(p.batch * p.Hkv * ((cols + 7) / 8))), dim3(256), 0, s, p);
  }
  return hipGetLastError();
}

}  // namespace scalify
