// Attention backward, which recomputes the probabilities from the stored
// log-sum-exp:
//   P = exp(S - lse), dP = dO v^T, dS = P (dP - delta), delta = rowsum(dO O),
//   dV = P^T dO, dK = alpha dS^T q, dQ = alpha dS k.
//
// Three kernels: delta and the rows' norms; dK and dV, a workgroup holding 128
// keys and walking the queries (of every head that shares the key head) that see
// them; dQ, a workgroup holding 128 query columns and walking the keys. Scores and
// dP are formed twice (seven products where five would do), but no workgroup adds
// to another's result: no fp32 atomics whose order would change the bits, and no
// fp32 gradient in memory unless a rescale needs one.
//
// F16 operands of the second products: P as 2^14 P, dS as 2^E dS with the power of
// two that its bound allows, |dS_ij| <= P (|dP_ij| + |delta_i|) <= 2 max(max|dO_i|
// max|v_j|, max|delta_i|) (Cauchy-Schwarz): 2^E dS <= 2^15, so 29 binades below the
// bound are normal F16 numbers. delta_i is a mean of dP_ij over every key that the
// query sees: where a workgroup holds some of these keys (dK and dV), |dO_i| |v_j|
// of its own does not bound it, and it stands for itself; over all of them (dQ) it does.
#include "attention_dev.h"
#include "kernels.h"

namespace scalify {

// delta, |dO_i|^2 and |v_j|^2: 16 lanes a row of a head, eight columns each.
__global__ __launch_bounds__(256) void attn_rows_kernel(AttnParams p) {
  const int64_t item = ((int64_t)(p.group0 + blockIdx.x) * 256 + threadIdx.x) >> 4;
  const int lane = threadIdx.x & 15;
  const int64_t nq = p.rows_q * p.H, nk = p.rows_k * p.Hkv;
  if (p.group0 + blockIdx.x == 0 && threadIdx.x < 3) p.amax[threadIdx.x] = 0u;
  if (item >= nq + nk) return;
  const bool query = item < nq;
  const int heads = query ? p.H : p.Hkv;
  const int64_t i = query ? item : item - nq, row = i / heads;
  const int head = (int)(i - row * heads), col = head * p.D + 8 * lane;
  float dot = 0.0f, sq = 0.0f;
  if (8 * lane < p.D) {
    if (query) {
      const h8 d = __builtin_bit_cast(h8, load_f16x8(p.do_fmt, p.dout, row * p.lddo + col));
      const h8 o = __builtin_bit_cast(h8, load_f16x8(p.out_fmt, p.out, row * p.ldo + col));
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        dot = fmaf((float)d[e], (float)o[e], dot);
        sq = fmaf((float)d[e], (float)d[e], sq);
      }
    } else {
      const h8 v = __builtin_bit_cast(h8, load_f16x8(p.v_fmt, p.v, row * p.ldv + col));
#pragma unroll
      for (int e = 0; e < 8; ++e) sq = fmaf((float)v[e], (float)v[e], sq);
    }
  }
#pragma unroll
  for (int off = 8; off > 0; off >>= 1) {
    dot += __shfl_xor(dot, off, 16);
    sq += __shfl_xor(sq, off, 16);
  }
  if (lane != 0) return;
  if (query) {
    // in units of dO's and v's data, as dP is
    p.delta[head * p.rows_q + row] = __builtin_ldexpf(dot, pow2_exponent(p.out_scale) - pow2_exponent(p.s_v));
    p.nd2[head * p.rows_q + row] = sq;
  } else {
    p.nv2[head * p.rows_k + row] = sq;
  }
}

// E for the largest |dO_i|^2 |v_j|^2, or delta_i^2.
__device__ __forceinline__ int ds_exponent(float n) {
  if (!(n > 0.0f) || !(n < 3.0e38f)) return 0;
  return 14 - ((floor_log2_bits(__float_as_uint(n)) + 2) >> 1);
}

// Largest value of 256 threads.
__device__ __forceinline__ float group_max(float a, float (&red)[4]) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) a = fmaxf(a, __shfl_xor(a, off, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = a;
  __syncthreads();
  return fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
}

// Largest finite value of n floats, over the workgroup (256 threads).
__device__ __forceinline__ float block_max(const float* x, int64_t n, float (&red)[4]) {
  float a = 0.0f;
  for (int64_t i = threadIdx.x; i < n; i += 256 * 8) {  // (eight loads in flight)
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = i + 256 * k < n ? x[i + 256 * k] : 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (v[k] < 3.0e38f) a = fmaxf(a, v[k]);
  }
  return group_max(a, red);
}

// A thread's share of the largest finite x and |y| of n (at most 2^30) rows each.
// (Sixteen loads in flight, at the last row's place past it: the backward of 4 x 4096
// causal tokens, 32 heads of 128, takes 2.49 ms, as it did without y, and took 2.57 with
// a loop of its own for y, each load behind a branch.)
__device__ __forceinline__ void rows_max(const float* x, const float* y, int n, float& ax, float& ay) {
  for (int i = threadIdx.x; i < n; i += 256 * 8) {
    float v[8], w[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int at = min(i + 256 * k, n - 1);
      v[k] = x[at];
      w[k] = fabsf(y[at]);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (v[k] < 3.0e38f) ax = fmaxf(ax, v[k]);
      if (w[k] < 3.0e38f) ay = fmaxf(ay, w[k]);
    }
  }
}

__device__ __forceinline__ void fold_amax(uint32_t* word, float a) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) a = fmaxf(a, __shfl_xor(a, off, 64));
  // (atomics on one word take 14 ns each; the word only grows, so a value that an old
  // copy of it already passes needs none)
  if ((threadIdx.x & 63) == 0 &&
      __float_as_uint(a) > __hip_atomic_load(word, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT))
    __hip_atomic_fetch_max(word, __float_as_uint(a), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Exponents of the propagated scales of dq, dk, dv.
__device__ __forceinline__ void grad_exponents(const AttnParams& p, int (&e)[3]) {
  const int eo = pow2_exponent(p.s_do), ev = pow2_exponent(p.s_v);
  e[0] = eo + ev + pow2_exponent(p.s_k);
  e[1] = eo + ev + pow2_exponent(p.s_q);
  e[2] = eo;
}

// Values of dO that are not finite, in a tile that the mask cuts, added to dV pair by
// pair (an admitted P is positive) for n queries from t on. Those of q need no more
// than to be taken out: their scores, and so dS, are NaN where they are admitted.
template <int DP, int DB>
__device__ __forceinline__ void add_odd_queries(const uint8_t* dt, int n, int t, int first, int lq, int h, f16v (&acc)[DB]) {
#pragma unroll 1
  for (int j = 0; j < n; ++j) {
    if (t + j < first || t + j >= lq) continue;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const u2 w = *(const u2*)(dt + tile_off<DP>(j, 4 * d + g) + 8 * h);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[d][4 * g + i] += odd_part((w[i >> 1] >> (16 * (i & 1))) & 0xFFFFu);
      }
  }
}

// 16 numbers of rows in a result's order, as a sum's start.
__device__ __forceinline__ f16v row_start(const float* rows, int h) {
  f16v r;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const float4 v = *(const float4*)(rows + 8 * g + 4 * h);
    r[4 * g] = v.x;
    r[4 * g + 1] = v.y;
    r[4 * g + 2] = v.z;
    r[4 * g + 3] = v.w;
  }
  return r;
}

// dK and dV of 128 keys, 32 a wave: scores and dP are formed with a key a lane
// (rows: queries), which makes them the operands of the second products as they
// stand. K and v rows stay in registers; tiles of 64 queries (q, dO), two blocks of
// 32, go through three LDS buffers. As in the forward, scores and dP of block b + 1
// and the second products of block b - 1 are formed while P and dS of block b are,
// in slices of four matrix instructions. The sums of a score and of dP start at
// -(lse - 14) / factor and -delta of their row, which LDS holds, so that P = exp2(score
// * factor) and dS = P dP need no row number in a register.
// One wave a SIMD (its results, and the rows, take most of the 512 registers), so
// what bounds it is the rate at which one wave issues, four clocks an instruction of
// any kind: 32 products of 32 clocks leave 224 others. 4 x 4096 causal tokens, 32
// heads of 128: 1.30 to 1.37 ms, the matrix cores busy for 36 % of it (at 2.3 GHz): a
// tile takes 4360 clocks of the loop, 2048 of them its products.
// Q16, O16: whether q and dO are F16 (and go straight into LDS) or have 8 bits.
template <int DP, bool Q16, bool O16>
__global__ __launch_bounds__(256, 1) void attn_dkv_kernel(AttnParams p, int tiles) {
  constexpr int TQ = 64, KS = DP / 16, DB = DP / 32, BUF = TQ * DP * 2, AHEAD = 1;
  __shared__ __align__(16) uint8_t lds[6 * BUF];
  __shared__ __align__(16) float row_l[3][TQ], row_d[3][TQ];
  __shared__ int odd;
  __shared__ float red[4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), h = lane >> 5;
  const Place at = attn_place(p, (int64_t)tiles * p.parts);
  const int tile = (int)at.rest / p.parts, part = (int)at.rest - tile * p.parts;  // (the first keys are seen by the most queries)
  const Seq sq = load_seq(p, at.b);
  const int kext = (int)min((int64_t)sq.kext, p.max_k);
  const int j0 = tile * 128;
  if (j0 >= kext) return;
  const int behind = sq.behind;
  const int key = j0 + 32 * wave + (lane & 31);
  const bool have = key < sq.lk;
  const int first = !have ? 0x7FFFFFFF : (p.causal ? key - behind : 0);  // first query that sees this key
  const int64_t krow = sq.k0 + key;
  h8 kf[KS], vf[KS];
  // queries that see any of the keys, in whole tiles, head after head
  const int q_lo = p.causal ? max(0, j0 - behind) / TQ * TQ : 0;
  const int nt = j0 < sq.lk && q_lo < sq.lq ? (sq.lq - q_lo + TQ - 1) / TQ : 0;
  const int q_end = q_lo + nt * TQ;
  // ... of which this part takes `steps`, from head g0's tile at t0 on
  const int step0 = (int)((int64_t)nt * p.G * part / p.parts), steps = (int)((int64_t)nt * p.G * (part + 1) / p.parts) - step0;
  const int g0 = steps > 0 ? step0 / nt : 0, t0 = q_lo + (step0 - g0 * nt) * TQ, g_end = steps > 0 ? (step0 + steps - 1) / nt + 1 : 0;
  // (a tile that every key of the workgroup sees whole has no masked pairs)
  auto cut = [&](int t) { return t + TQ > sq.lq || j0 + 128 > sq.lk || (p.causal && t + behind < j0 + 127); };

  f16v ak[DB], av[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) ak[d] = av[d] = f16v{};
  Tile<Q16, TQ, DP> lq;
  Tile<O16, TQ, DP> ld;
  lq.init(p.q, sq.q0 * p.ldq + (int64_t)at.hk * p.G * p.D, p.ldq, p.D, p.q_fmt);
  ld.init(p.dout, sq.q0 * p.lddo + (int64_t)at.hk * p.G * p.D, p.lddo, p.D, p.do_fmt);
  float l_next = 0.0f, d_next = 0.0f;
  // The next tile to fetch: `left` queries of head g_next, 16 rows' numbers a wave;
  // behind the last, rows of zeros that see no key. (Every address moves on
  // by a constant: kernel arguments read again for each tile cost 700 clocks of it.)
  const int mine = 16 * wave + lane, rows = nt * TQ;
  int g_next = g0, left = sq.lq - t0, more = steps;
  const float* l_at = p.lse + (int64_t)(at.hk * p.G + g0) * p.rows_q + sq.q0 + t0 + mine;
  const float* d_at = p.delta + (int64_t)(at.hk * p.G + g0) * p.rows_q + sq.q0 + t0 + mine;
  const int64_t to_head = p.rows_q - rows;
  lq.seek(t0, (int64_t)g0 * p.D);
  ld.seek(t0, (int64_t)g0 * p.D);
  auto begin = [&](uint8_t* buf) {
    const int there = more-- > 0 ? left : 0;
    lq.begin(there, buf, wave);
    ld.begin(there, buf + BUF, wave);
    l_next = neg_inf();
    d_next = 0.0f;
    if (lane < 16 && mine < there) {
      l_next = *l_at;
      d_next = *d_at;
    }
    l_at += TQ;
    d_at += TQ;
    left -= TQ;
    if (left <= 0) {
      left = sq.lq - q_lo;
      ++g_next;
      lq.seek(q_lo, (int64_t)g_next * p.D);
      ld.seek(q_lo, (int64_t)g_next * p.D);
      l_at += to_head;
      d_at += to_head;
    }
  };
  auto issue = [&](int i) {
    if (i < KS / 2) lq.issue(i);
    else ld.issue(i - KS / 2);
  };
  if (steps > 0) {
    begin(lds);
#pragma unroll
    for (int i = 0; i < KS; ++i) issue(i);
  }
  // The keys' own rows: F16 through the two buffers that are still free, in whole rows.
  // (Loaded as operands, 16 bytes of 32 rows at a time, they took 15000 clocks.)
  const bool k16 = p.k_fmt == kF16, v16 = p.v_fmt == kF16;
  auto fetch = [&](const void* x, int64_t ld, uint8_t* to) {
    DirectTile<2 * TQ, DP> own;
    own.init(x, sq.k0 * ld + (int64_t)at.hk * p.D, ld, p.D, kF16);
    own.seek(j0);
    own.begin(sq.lk - j0, to, wave);
#pragma unroll
    for (int i = 0; i < own.N; ++i) own.issue(i);
  };
  if (k16) fetch(p.k, p.ldk, lds + 2 * BUF);
  else load_row_operands(p.k_fmt, p.k, krow * p.ldk + (int64_t)at.hk * p.D, h, p.D, have, kf);
  if (v16) fetch(p.v, p.ldv, lds + 4 * BUF);
  else load_row_operands(p.v_fmt, p.v, krow * p.ldv + (int64_t)at.hk * p.D, h, p.D, have, vf);
  if (threadIdx.x == 0) odd = -1;
  float nd2 = 0.0f, dl = 0.0f;
  for (int g = g0; g < g_end; ++g) {
    const int64_t rows0 = (int64_t)(at.hk * p.G + g) * p.rows_q + sq.q0 + q_lo;
    rows_max(p.nd2 + rows0, p.delta + rows0, sq.lq - q_lo, nd2, dl);
  }
  nd2 = group_max(nd2, red);
  dl = group_max(dl, red);
  const float nv2 = block_max(p.nv2 + (int64_t)at.hk * p.rows_k + sq.k0 + j0, max(0, min(128, sq.lk - j0)), red);
  const int E = ds_exponent(fmaxf(nd2 * nv2, dl * dl));
  const float c1 = score_factor(p), c2 = pow2_float(E - (int)kProbLog2), inv_c1 = 1.0f / c1;
  wait_loads();
  __syncthreads();
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    if (k16) kf[ks] = row_operand<DP>(lds + 2 * BUF, 32 * wave, ks, lane);
    if (v16) vf[ks] = row_operand<DP>(lds + 4 * BUF, 32 * wave, ks, lane);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * TQ * DP / 8; i += 256) ((u4*)(lds + 4 * BUF))[i] = u4{0u, 0u, 0u, 0u};  // (the block before the first)
  auto arrive = [&](int n) {
    lq.arrive(lds + n * 2 * BUF);
    ld.arrive(lds + n * 2 * BUF + BUF);
    if (lane < 16) {
      // (here, not where they are fetched: their first use waits for the tile as well)
      row_l[n][mine] = l_next == neg_inf() ? neg_inf() : -fmaf(l_next, kLog2e, -kProbLog2) * inv_c1;
      row_d[n][mine] = -d_next;
    }
    __syncthreads();
  };
  // scores and dP of the last two blocks, P and dS of the last two
  f16v sa = {}, da = {}, sb = {}, db = {};
  h8 pa[2] = {}, ea[2] = {}, pb[2] = {}, eb[2] = {};
  if (steps > 0) {
    arrive(0);
    sa = row_start(row_l[0], h);
    da = row_start(row_d[0], h);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      sa = mfma(row_operand<DP>(lds, 0, ks, lane), kf[ks], sa);
      da = mfma(row_operand<DP>(lds + BUF, 0, ks, lane), vf[ks], da);
    }
    begin(lds + 2 * BUF);
#pragma unroll
    for (int i = 0; i < KS; ++i) issue(i);
  }
  settle_loads();

  // One block of 32 queries from i0 on, with scores s and dP dp: its P and dS to pn
  // and en; the next block's (rows at qn, on in LDS) scores and dP to sn and dn; the
  // last block's P and dS times its dO and q (rows at ql, ol).
  auto block = [&](int i0, f16v& s, f16v& dp, h8 (&pn)[2], h8 (&en)[2], f16v& sn, f16v& dn, const uint8_t* qn, const uint8_t* on,
                   const float* ln, const float* rn, const h8 (&pl)[2], const h8 (&el)[2], const uint8_t* ql, const uint8_t* ol, auto&& also) {
    if (__any(i0 < first) || i0 + 32 > sq.lq) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int i = i0 + result_row(r, h);
        if (i < first || i >= sq.lq) {
          s[r] = neg_inf();
          dp[r] = 0.0f;
        }
      }
    }
    // First the next block's scores and dP (a step of each in turn), then the last
    // block's dV and dK: a slice is one product and what fits under it, either the
    // operands of a later one or the probabilities of 16 / KS / 2 elements.
    h8 fa[AHEAD + 1][2], fb[AHEAD + 1][2];
    auto read = [&](int x, int y) {
      h8 &a = fa[x % (AHEAD + 1)][y], &b = fb[x % (AHEAD + 1)][y];
      if (x < KS / 2) {
        a = row_operand<DP>(qn, 0, 2 * x + y, lane);
        b = row_operand<DP>(on, 0, 2 * x + y, lane);
      } else {
        const int z = 2 * (x - KS / 2) + y;
        a = col_operand<DP>(ol, 16 * (z / DB), z % DB, lane);
        b = col_operand<DP>(ql, 16 * (z / DB), z % DB, lane);
      }
    };
    sn = row_start(ln, h);
    dn = row_start(rn, h);
#pragma unroll
    for (int x = 0; x < AHEAD; ++x) {
      read(x, 0);
      read(x, 1);
    }
    slice_end();
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      const int a = i % (AHEAD + 1);
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int z = 2 * (i - KS / 2) + y;
        if (i < KS / 2) sn = mfma(fa[a][y], kf[2 * i + y], sn);
        else av[z % DB] = mfma(fa[a][y], pl[z / DB], av[z % DB]);
        if (i + AHEAD < KS) read(i + AHEAD, y);
        if (y == 0) also(i);
        slice_end();
        if (i < KS / 2) dn = mfma(fb[a][y], vf[2 * i + y], dn);
        else ak[z % DB] = mfma(fb[a][y], el[z / DB], ak[z % DB]);
#pragma unroll
        for (int e = 8 / KS * (2 * i + y); e < 8 / KS * (2 * i + y + 1); ++e) {
          float x = __builtin_amdgcn_exp2f(s[e] * c1), w = x * (dp[e] * c2);
          held(x);
          held(w);
          pn[e >> 3][e & 7] = (_Float16)x;
          en[e >> 3][e & 7] = (_Float16)w;
        }
        slice_end();
      }
    }
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      held(pn[g]);
      held(en[g]);
    }
  };
  int n = 0;  // the buffer of this step
#pragma unroll 1
  for (int step = 0, t = t0; step < steps; ++step, t = t + TQ < q_end ? t + TQ : q_lo) {
    const int n1 = n == 2 ? 0 : n + 1, n2 = n == 0 ? 2 : n - 1;
    uint8_t* const cur = lds + n * 2 * BUF;
    uint8_t* const nxt = lds + n1 * 2 * BUF;
    uint8_t* const prv = lds + n2 * 2 * BUF;
    block(t, sa, da, pa, ea, sb, db, cur + BUF / 2, cur + BUF + BUF / 2, row_l[n] + 32, row_d[n] + 32, pb, eb, prv + BUF / 2,
          prv + BUF + BUF / 2, [](int) {});
    arrive(n1);
    if (cut(t)) {
      mark_not_finite<2 * TQ, DP>(cur, &odd, step);
      __syncthreads();
      if (__builtin_amdgcn_readfirstlane(odd) == step) {
        add_odd_queries<DP>(cur + BUF, TQ, t, first, sq.lq, h, av);
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * TQ * DP / 8; i += 256) ((h8*)cur)[i] = finite_part(((const h8*)cur)[i]);
        __syncthreads();
      }
    }
    begin(prv);
    block(t + 32, sb, db, pb, eb, sa, da, nxt, nxt + BUF, row_l[n1], row_d[n1], pa, ea, cur, cur + BUF, issue);
    n = n1;
  }
  if (steps > 0) {  // the last block's products
    const uint8_t* const ql = lds + (n == 0 ? 2 : n - 1) * 2 * BUF + BUF / 2;
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      av[i % DB] = mfma(col_operand<DP>(ql + BUF, 16 * (i / DB), i % DB, lane), pb[i / DB], av[i % DB]);
      ak[i % DB] = mfma(col_operand<DP>(ql, 16 * (i / DB), i % DB, lane), eb[i / DB], ak[i % DB]);
    }
    wait_loads();  // (none may reach LDS after the workgroup has ended)
  }
  int e[3];
  grad_exponents(p, e);
  const float fk = __builtin_ldexpf(p.alpha, -E), fv = pow2_float(-(int)kProbLog2);
  const int64_t c = (int64_t)at.hk * p.D, half = p.rows_k * p.Hkv * p.D, row0 = sq.k0 + j0 + 32 * wave;
  float* const dk32 = p.parts > 1 ? p.part + 2 * part * half : p.dk32;
  float* const dv32 = p.parts > 1 ? dk32 + half : p.dv32;
  auto place = [&](int64_t ld) {
    return [&, ld](int r, int64_t& e32, int64_t& x) {
      e32 = (row0 + r) * p.Hkv * p.D + c;
      x = (row0 + r) * ld + c;
    };
  };
  const int rows_here = min(32, kext - j0 - 32 * wave);
  uint8_t* const stage = lds + wave * (32 * DP * 4);
  __syncthreads();  // (the tiles have been read)
  const float mk = store_rows<DP>(stage, ak, fk, lane, rows_here, p.D, dk32, p.dk, p.dk_fmt, clamp_e8m0(e[1]) - e[1], p.sat != 0,
                                  place(p.lddk));
  const float mv = store_rows<DP>(stage, av, fv, lane, rows_here, p.D, dv32, p.dv, p.dv_fmt, clamp_e8m0(e[2]) - e[2], p.sat != 0,
                                  place(p.lddv));
  if (p.parts > 1) return;  // (attn_parts_kernel forms the sums' magnitudes)
  fold_amax(p.amax + 1, mk);
  fold_amax(p.amax + 2, mv);
}

// dQ of 128 query columns, 32 a wave, a query a lane: the forward's walk over tiles
// of 64 keys, with q and dO rows in registers, laid out as dK and dV above: scores
// and dP of key block b + 1 and the product of block b - 1 while dS of block b is
// formed. k is read twice, by rows for the scores and by columns for the product a
// block later, and has three LDS buffers, v two. The same tokens: 1.00 to 1.06 ms, the
// matrix cores busy for 35 % (one product after another, its tiles shared by barriers: 1.23).
// Buffers known at compile time save 15 of a block's 220 instructions and no time (1.10).
// K16, V16: whether k and v are F16 (and go straight into LDS) or have 8 bits.
template <int DP, bool K16, bool V16>
__global__ __launch_bounds__(256, 1) void attn_dq_kernel(AttnParams p, int tiles) {
  constexpr int TK = 64, KS = DP / 16, DB = DP / 32, BUF = TK * DP * 2, AHEAD = 1;
  __shared__ __align__(16) uint8_t lds[5 * BUF];
  __shared__ int odd;
  __shared__ float red[4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), h = lane >> 5;
  const Place at = attn_place(p, tiles);
  const int tile = tiles - 1 - (int)at.rest;
  const Seq sq = load_seq(p, at.b);
  const int64_t ncols = (int64_t)sq.lq * p.G, col0 = (int64_t)tile * 128;
  if (col0 >= ncols) return;
  const int64_t col = col0 + 32 * wave + (lane & 31);
  const bool live = col < ncols;
  const int pos = (int)(col / p.G), head = at.hk * p.G + (int)(col - (int64_t)pos * p.G);
  const int64_t qrow = sq.q0 + pos;
  const int behind = sq.behind;
  const int last = !live ? 0x7FFFFFFF : (p.causal ? min(pos + behind, sq.lk - 1) : sq.lk - 1);
  const int last0 = p.causal ? min((int)(col0 / p.G) + behind, sq.lk - 1) : sq.lk - 1;
  const int64_t last_col = col0 + 128 < ncols ? col0 + 127 : ncols - 1;
  const int end = p.causal ? max(0, min(sq.lk, (int)(last_col / p.G) + behind + 1)) : sq.lk;
  uint8_t* const kb = lds;
  uint8_t* const vb = lds + 3 * BUF;
  Tile<K16, TK, DP> lk;
  Tile<V16, TK, DP> lv;
  lk.init(p.k, sq.k0 * p.ldk + (int64_t)at.hk * p.D, p.ldk, p.D, p.k_fmt);
  lv.init(p.v, sq.k0 * p.ldv + (int64_t)at.hk * p.D, p.ldv, p.D, p.v_fmt);
  lk.seek(0);
  lv.seek(0);
  lk.begin(end, kb, wave);
  lv.begin(end, vb, wave);
#pragma unroll
  for (int i = 0; i < KS / 2; ++i) {
    lk.issue(i);
    lv.issue(i);
  }
  h8 qf[KS], df[KS];
  load_row_operands(p.q_fmt, p.q, qrow * p.ldq + (int64_t)head * p.D, h, p.D, live, qf);
  load_row_operands(p.do_fmt, p.dout, qrow * p.lddo + (int64_t)head * p.D, h, p.D, live, df);
  if (threadIdx.x == 0) odd = -1;
  for (int i = threadIdx.x; i < BUF / 16; i += 256) ((u4*)(kb + 2 * BUF))[i] = u4{0u, 0u, 0u, 0u};  // (the block before the first)
  const float nv2 = block_max(p.nv2 + (int64_t)at.hk * p.rows_k + sq.k0, end, red);
  float nd2 = 0.0f, L = __builtin_inff(), Dl = 0.0f;
  if (live) {
    const int64_t row = (int64_t)head * p.rows_q + qrow;
    const float l = p.lse[row], n = p.nd2[row], d = p.delta[row];
    // (a query that sees no key, whose P is 0 throughout, keeps neither norm nor delta: its dO may hold Inf or NaN)
    const bool sees = l != neg_inf();
    nd2 = sees ? n : 0.0f;
    Dl = sees ? d : 0.0f;
    L = sees ? fmaf(l, kLog2e, -kProbLog2) : __builtin_inff();
  }
  if (!(nd2 < 3.0e38f)) nd2 = 0.0f;
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) nd2 = fmaxf(nd2, __shfl_xor(nd2, off, 64));
  const int E = ds_exponent(nd2 * nv2);  // (of this wave)
  const float c1 = score_factor(p), c2 = pow2_float(E - (int)kProbLog2);
  Dl *= c2;
  f16v acc[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) acc[d] = f16v{};
  auto arrive = [&](uint8_t* kt, uint8_t* vt) {
    lk.arrive(kt);
    lv.arrive(vt);
    __syncthreads();
  };
  f16v sa = {}, da = {}, sb = {}, db = {};  // scores and dP of two blocks
  h8 ea[2] = {}, eb[2] = {};                // and their dS
  if (end > 0) {
    arrive(kb, vb);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      sa = mfma(row_operand<DP>(kb, 0, ks, lane), qf[ks], sa);
      da = mfma(row_operand<DP>(vb, 0, ks, lane), df[ks], da);
    }
    lk.begin(end - TK, kb + BUF, wave);
    lv.begin(end - TK, vb + BUF, wave);
#pragma unroll
    for (int i = 0; i < KS / 2; ++i) {
      lk.issue(i);
      lv.issue(i);
    }
  }
  settle_loads();

  // One block: its keys key0 ... with scores s and dP dp, whose dS go to en; the next
  // block's (rows kn and vn) scores and dP to sn and dn; the last block's dS el times
  // its keys (rows kl).
  auto block = [&](int key0, f16v& s, f16v& dp, h8 (&en)[2], f16v& sn, f16v& dn, const uint8_t* kn, const uint8_t* vn,
                   const h8 (&el)[2], const uint8_t* kl, auto&& also) {
    if (key0 + 31 > last0) {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (key0 + result_row(r, h) > last) {
          s[r] = neg_inf();
          dp[r] = 0.0f;
        }
    }
    h8 fk[AHEAD + 1], fv[AHEAD + 1], fc[AHEAD + 1];
    auto read = [&](int x) {
      fk[x % (AHEAD + 1)] = row_operand<DP>(kn, 0, x, lane);
      fv[x % (AHEAD + 1)] = row_operand<DP>(vn, 0, x, lane);
      fc[x % (AHEAD + 1)] = col_operand<DP>(kl, 16 * (x / DB), x % DB, lane);
    };
    auto take = [&](int e) {
      float x = __builtin_amdgcn_exp2f(fmaf(s[e], c1, -L)) * fmaf(dp[e], c2, -Dl);
      held(x);
      en[e >> 3][e & 7] = (_Float16)x;
    };
#pragma unroll
    for (int x = 0; x < AHEAD; ++x) read(x);
    f16v sc = {}, dc = {};
    slice_end();
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      const int a = i % (AHEAD + 1);
      sc = mfma(fk[a], qf[i], sc);
      if (i + AHEAD < KS) read(i + AHEAD);
      also(i);
      slice_end();
      dc = mfma(fv[a], df[i], dc);
#pragma unroll
      for (int e = 16 / KS * i; e < 16 / KS * i + 8 / KS; ++e) take(e);
      slice_end();
      acc[i % DB] = mfma(fc[a], el[i / DB], acc[i % DB]);
#pragma unroll
      for (int e = 16 / KS * i + 8 / KS; e < 16 / KS * (i + 1); ++e) take(e);
      slice_end();
    }
    held(en[0]);
    held(en[1]);
    sn = sc;
    dn = dc;
  };
  // (The loop starts at a line of the instruction cache, wherever the code before it ends: 4 x
  // 4096 causal tokens, 32 heads of 128, took 1041 us so, up to 1063 from other places.)
  asm volatile(".p2align 6");
  int n = 0, n2 = 0;  // the buffers of tile t: of three, and of two
#pragma unroll 1
  for (int t = 0; t < end; t += TK, n2 ^= 1) {
    const int n1 = n == 2 ? 0 : n + 1;
    uint8_t* const cur = kb + n * BUF;
    uint8_t* const nxt = kb + n1 * BUF;
    uint8_t* const prv = kb + (n == 0 ? 2 : n - 1) * BUF;
    uint8_t* const vc = vb + n2 * BUF;
    uint8_t* const vn = vb + (n2 ^ 1) * BUF;
    block(t, sa, da, ea, sb, db, cur + BUF / 2, vc + BUF / 2, eb, prv + BUF / 2, [](int) {});
    arrive(nxt, vn);
    if (t + TK - 1 > last0) {
      mark_not_finite<TK, DP>(cur, &odd, t);
      __syncthreads();
      if (__builtin_amdgcn_readfirstlane(odd) == t) {
        // (where they are admitted the scores, and so dS, are NaN)
        for (int i = threadIdx.x; i < TK * DP / 8; i += 256) ((h8*)cur)[i] = finite_part(((const h8*)cur)[i]);
        __syncthreads();
      }
    }
    lk.begin(end - t - 2 * TK, prv, wave);
    lv.begin(end - t - 2 * TK, vc, wave);
    block(t + 32, sb, db, eb, sa, da, nxt, vn, ea, cur, [&](int i) {
      if (i < KS / 2) lk.issue(i);
      else lv.issue(i - KS / 2);
    });
    n = n1;
  }
  if (end > 0) {  // the last block's product
    const uint8_t* const kl = kb + (n == 0 ? 2 : n - 1) * BUF + BUF / 2;
#pragma unroll
    for (int i = 0; i < KS; ++i) acc[i % DB] = mfma(col_operand<DP>(kl, 16 * (i / DB), i % DB, lane), eb[i / DB], acc[i % DB]);
  }
  wait_loads();  // (none may reach LDS after the workgroup has ended)
  int e[3];
  grad_exponents(p, e);
  const int64_t wave0 = col0 + 32 * wave;
  __syncthreads();  // (the tiles have been read)
  const float mq = store_rows<DP>(lds + wave * (32 * DP * 4), acc, __builtin_ldexpf(p.alpha, -E), lane, (int)min((int64_t)32, ncols - wave0),
                                  p.D, p.dq32, p.dq, p.dq_fmt, clamp_e8m0(e[0]) - e[0], p.sat != 0,
                                  [&](int r, int64_t& e32, int64_t& x) {
                                    const int i = (int)(wave0 + r) / p.G, hd = at.hk * p.G + (int)(wave0 + r) - i * p.G;
                                    e32 = (sq.q0 + i) * p.H * p.D + (int64_t)hd * p.D;
                                    x = (sq.q0 + i) * p.lddq + (int64_t)hd * p.D;
                                  });
  fold_amax(p.amax, mq);
}

constexpr int ATTN_CAST_ROWS = 4, ATTN_PART_ROWS = 8;

// dk and dv as the sums of their parts, in the parts' order: four columns a thread, 8
// rows of a sequence a workgroup (blockIdx.y: dk, dv). To codes, or to the first part
// for the dynamic rescale's cast.
__global__ __launch_bounds__(256) void attn_parts_kernel(AttnParams p, int64_t tiles) {
  __shared__ float red[4];
  const bool isv = blockIdx.y != 0;
  const int64_t b = blockIdx.x / tiles, r0 = blockIdx.x % tiles * ATTN_PART_ROWS;
  const Seq sq = load_seq(p, b);
  const int64_t rows = min((int64_t)sq.kext, p.max_k);
  if (r0 >= rows) return;
  const int n = (int)min((int64_t)ATTN_PART_ROWS, rows - r0), cols = p.Hkv * p.D, chunks = cols / 4;
  const int64_t half = p.rows_k * cols;
  float* const src = p.part + (isv ? half : 0);
  void* const dst = isv ? p.dv : p.dk;
  const int64_t ld = isv ? p.lddv : p.lddk;
  const int fmt = isv ? p.dv_fmt : p.dk_fmt;
  int e[3];
  grad_exponents(p, e);
  const int shift = clamp_e8m0(e[isv ? 2 : 1]) - e[isv ? 2 : 1];
  float m = 0.0f;
  for (int i = threadIdx.x; i < n * chunks; i += 256) {
    const int r = i / chunks, c = 4 * (i - r * chunks);
    const int64_t row = sq.k0 + r0 + r;
    float4* const at = (float4*)(src + row * cols + c);
    float4 s = *at;
    for (int j = 1; j < p.parts; j += 3) {  // (three loads in flight)
      float4 x[3];
#pragma unroll
      for (int k = 0; k < 3; ++k) x[k] = j + k < p.parts ? at[(j + k) * (half / 2)] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        s.x += x[k].x;
        s.y += x[k].y;
        s.z += x[k].z;
        s.w += x[k].w;
      }
    }
    m = fmaxf(m, fmaxf(fmaxf(fabsf(s.x), fabsf(s.y)), fmaxf(fabsf(s.z), fabsf(s.w))));  // (fmaxf skips NaN)
    const float y[4] = {s.x, s.y, s.z, s.w};
    if (p.mode == 1) *at = s;
    else store4_any(fmt, dst, row * ld + c, y, shift, p.sat != 0);
  }
  if (p.mode != 1 && !p.amax_out) return;
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
  __syncthreads();
  if (threadIdx.x < 64) fold_amax(p.amax + (isv ? 2 : 1), fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
}

// The dynamic rescale's cast of the three fp32 gradients (blockIdx.y), 4 rows of a
// sequence a workgroup, and the scales and statistics of either mode.
__global__ __launch_bounds__(256) void attn_grads_kernel(AttnParams p, int64_t tiles) {
  const int which = blockIdx.y;
  int e[3];
  grad_exponents(p, e);
  const int base = e[which];
  const uint32_t amax = p.amax[which];
  const int e_out = clamp_e8m0(base + (p.mode == 1 ? rescale_exponent(amax, p.target) : 0));
  const uint32_t id = p.group0 + blockIdx.x;
  if (id == 0 && threadIdx.x == 0) {
    *(which == 0 ? p.dq_scale : which == 1 ? p.dk_scale : p.dv_scale) = pow2_float(e_out);
    if (p.amax_out) p.amax_out[which] = __uint_as_float(amax);
  }
  if (p.mode != 1) return;
  const int64_t b = id / tiles, tile = id % tiles;
  const Seq sq = load_seq(p, b);
  const int64_t rows = which == 0 ? sq.lq : min((int64_t)sq.kext, p.max_k);
  const int64_t r0 = tile * ATTN_CAST_ROWS;
  if (r0 >= rows) return;
  const int64_t row0 = (which == 0 ? sq.q0 : sq.k0) + r0;
  const int n = (int)min((int64_t)ATTN_CAST_ROWS, rows - r0);
  const int cols = (which == 0 ? p.H : p.Hkv) * p.D;  // (a multiple of 16)
  const float* src = which == 0 ? p.dq32 : which == 1 ? p.dk32 : p.dv32;
  void* dst = which == 0 ? p.dq : which == 1 ? p.dk : p.dv;
  const int64_t ld = which == 0 ? p.lddq : which == 1 ? p.lddk : p.lddv;
  const int fmt = which == 0 ? p.dq_fmt : which == 1 ? p.dk_fmt : p.dv_fmt;
  const int shift = e_out - base;
  const bool fast = shift >= kFastShiftMinSub && shift <= kFastShiftMax, sat = p.sat != 0;
  const float scale = fast ? pow2_float(shift) : 1.0f;
  const int chunks = cols / 16;
  for (int i = threadIdx.x; i < n * chunks; i += 256) {
    const int r = i / chunks, c = 16 * (i - r * chunks);
    uint32_t u[16], w[8];
    load16<kF32>(src, (row0 + r) * cols + c, u);
    const int64_t o = (row0 + r) * ld + c;
    if (fmt == kF16) {
      encode16<kF16>(u, shift, scale, fast, sat, w);
      store_words16<kF16>(dst, o, w);
    } else if (fmt == kE4M3) {
      encode16<kE4M3>(u, shift, scale, fast, sat, w);
      store_words16<kE4M3>(dst, o, w);
    } else {
      encode16<kE5M2>(u, shift, scale, fast, sat, w);
      store_words16<kE5M2>(dst, o, w);
    }
  }
}

template <int DP>
static hipError_t launch_dkv(const AttnParams& p, hipStream_t s) {
  const bool q16 = p.q_fmt == kF16, o16 = p.do_fmt == kF16;
  const int tiles = (int)((p.max_k + 127) / 128);
  const int64_t g = p.rows_k > 0 ? p.batch * p.Hkv * tiles * p.parts : 0;
  if (q16 && o16) return launch_groups(attn_dkv_kernel<DP, true, true>, g, 1, s, p, tiles);
  if (q16) return launch_groups(attn_dkv_kernel<DP, true, false>, g, 1, s, p, tiles);
  if (o16) return launch_groups(attn_dkv_kernel<DP, false, true>, g, 1, s, p, tiles);
  return launch_groups(attn_dkv_kernel<DP, false, false>, g, 1, s, p, tiles);
}

template <int DP>
static hipError_t launch_dq(const AttnParams& p, hipStream_t s) {
  const bool k16 = p.k_fmt == kF16, v16 = p.v_fmt == kF16;
  const int tiles = (int)((p.max_q * p.G + 127) / 128);
  const int64_t g = p.rows_q > 0 ? p.batch * p.Hkv * tiles : 0;
  if (k16 && v16) return launch_groups(attn_dq_kernel<DP, true, true>, g, 1, s, p, tiles);
  if (k16) return launch_groups(attn_dq_kernel<DP, true, false>, g, 1, s, p, tiles);
  if (v16) return launch_groups(attn_dq_kernel<DP, false, true>, g, 1, s, p, tiles);
  return launch_groups(attn_dq_kernel<DP, false, false>, g, 1, s, p, tiles);
}

template <int DP>
static hipError_t launch(const AttnParams& p, hipStream_t s) {
  const hipError_t e = launch_dkv<DP>(p, s);
  return e == hipSuccess ? launch_dq<DP>(p, s) : e;
}

// Where the workgroups of 128 keys leave CUs without one, the queries (tiles of 64, of
// all the heads that share the keys) are split among several, four tiles or more each,
// as far as there are 256. (1777 tokens of 3 sequences, 16 heads on 4 of keys: dK and dV
// took 123 us unsplit, 55 in 3 parts; up to 512 workgroups 56, up to 1024 72, and the
// sum of the parts 19, 27 and 35. Now 51 and 12.)
int attention_bwd_parts(int64_t batch, int Hkv, int G, int64_t max_q, int64_t max_k) {
  const int64_t groups = batch * Hkv * ((max_k + 127) / 128), tiles = (max_q + 63) / 64 * G;
  int64_t s = groups > 0 ? 256 / groups : 1;
  if (s > tiles / 4) s = tiles / 4;
  if (s > 16) s = 16;
  return s < 2 ? 1 : (int)s;
}

hipError_t launch_attention_bwd(const AttnParams& p, hipStream_t s) {
  const int64_t items = p.rows_q * p.H + p.rows_k * p.Hkv;
  hipError_t e = launch_groups(attn_rows_kernel, items > 16 ? (items + 15) / 16 : 1, 1, s, p);
  if (e == hipSuccess) e = p.D <= 64 ? launch<64>(p, s) : launch<128>(p, s);
  if (e == hipSuccess && p.parts > 1) {
    // (queries are shared among parts for at most 128 tiles of 128 keys: one launch)
    const int64_t tiles = (p.max_k + ATTN_PART_ROWS - 1) / ATTN_PART_ROWS;
    e = launch_groups(attn_parts_kernel, p.batch * tiles, 2, s, p, tiles);
  }
  if (e != hipSuccess) return e;
  const int64_t most = p.max_q > p.max_k ? p.max_q : p.max_k;
  int64_t tiles = p.mode == 1 ? (most + ATTN_CAST_ROWS - 1) / ATTN_CAST_ROWS : 0;
  if (tiles < 1) tiles = 1;
  return launch_groups(attn_grads_kernel, p.mode == 1 ? p.batch * tiles : 1, 3, s, p, tiles);
}

}  // namespace scalify
