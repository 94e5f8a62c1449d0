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
//   few (32 columns, which each wave holds, with tiles of keys of its own; the waves
//     are joined at the end): single tokens; bound by reading the cache.
// Where that leaves the device idle the keys of a sequence are split over
// workgroups, whose unnormalised results a second kernel joins.
#include "attention_dev.h"
#include "kernels.h"

namespace scalify {

// The forward keeps 2^10 p relative to the running maximum, which a score may pass
// by kSlack before it is moved (moving it multiplies every result, and with 32
// queries a wave some query would move it in most tiles): at most 2^15, and
// normal F16 numbers down to p = 2^-24.
constexpr float kRunLog2 = 10.0f, kSlack = 5.0f;

// A query a lane: where it is, and what it sees.
struct Query {
  int64_t row;
  int head, last;  // the last key it sees; a lane without a query sees every key (its result goes nowhere)
  bool live;
};
__device__ __forceinline__ Query query_at(const AttnParams& p, const Seq& sq, int hk, int64_t col, int64_t ncols) {
  Query q;
  q.live = col < ncols;
  const int pos = (int)(col / p.G);
  q.head = hk * p.G + (int)(col - (int64_t)pos * p.G);
  q.row = sq.q0 + pos;
  q.last = !q.live ? 0x7FFFFFFF : (p.causal ? min(pos + sq.behind, sq.lk - 1) : sq.lk - 1);
  return q;
}

// The keys of a workgroup: those that its last column sees, a split's share of
// them in whole tiles.
__device__ __forceinline__ void key_range(const AttnParams& p, const Seq& sq, int64_t last_col, int split, int tile, int& begin,
                                          int& end) {
  const int seen = p.causal ? max(0, min(sq.lk, (int)(last_col / p.G) + sq.behind + 1)) : sq.lk;
  const int share = ((seen + p.splits - 1) / p.splits + tile - 1) / tile * tile;
  begin = (int)min((int64_t)split * share, (int64_t)seen);
  end = min(seen, begin + share);
}

// Block d (32 columns) of a query's result: of every four registers the columns
// are consecutive.
__device__ __forceinline__ void store_result(const AttnParams& p, const f16v& o, const Query& q, int d, int h, float l, int split) {
  const float inv = 1.0f / l;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const int n = 32 * d + 8 * g + 4 * h;
    if (n >= p.D) continue;
    if (p.splits > 1) {
      *(float4*)(p.part_o + ((split * p.rows_q + q.row) * p.H + q.head) * (int64_t)p.D + n) =
          make_float4(o[4 * g], o[4 * g + 1], o[4 * g + 2], o[4 * g + 3]);
    } else {
      float y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = l == 0.0f ? 0.0f : o[4 * g + i] * inv;
      store4_any(p.out_fmt, p.out, q.row * p.ldo + (int64_t)q.head * p.D + n, y, 0, p.sat != 0);
    }
  }
}
__device__ __forceinline__ float log_sum(float m, float l) {
  return l == 0.0f ? neg_inf() : (m - kRunLog2 + __builtin_amdgcn_logf(l)) * kLn2;
}
__device__ __forceinline__ void store_row(const AttnParams& p, const Query& q, float m, float l, int split) {
  if (p.splits > 1) p.part_ml[(split * p.rows_q + q.row) * p.H + q.head] = make_float2(m, l);
  else if (p.lse) p.lse[(int64_t)q.head * p.rows_q + q.row] = log_sum(m, l);
}

// Scores (key0 + row, query) that the mask does not admit.
__device__ __forceinline__ void mask_scores(f16v& s, int key0, int h, int last) {
#pragma unroll
  for (int r = 0; r < 16; ++r)
    if (key0 + result_row(r, h) > last) s[r] = neg_inf();
}

// The running maximum, in powers of two, with scores up to `top` (of this lane's
// half, before their factor), and what the sum and the results have to be
// multiplied with. The maximum is moved only when a score is past it by more than
// kSlack: probabilities relative to it may then reach 2^kSlack, which F16 holds.
template <int DB>
__device__ __forceinline__ void run_max(float top, float c1, int h, float& m, float& l, f16v (&acc)[DB]) {
  top = fmaxf(top, other_half(top, h)) * c1;
  if (__any(top > m + kSlack)) {
    const float now = fmaxf(m, top);
    const float f = m == neg_inf() ? 1.0f : __builtin_amdgcn_exp2f(m - now);  // (so far nothing but infinities may have been added)
    m = now;
    l *= f;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[d][r] *= f;
  }
}
__device__ __forceinline__ float block_top(const f16v& s) {
  float top = s[0];
#pragma unroll
  for (int r = 1; r < 16; ++r) top = fmaxf(top, s[r]);  // (fmaxf skips NaN)
  return top;
}

// Values of v that are not finite, in a tile that the mask cuts, are added pair by
// pair (an admitted probability is positive, so its product with an infinity is
// that infinity) and then taken out of the tile. n rows from row0 on, keys key0 ...
template <int DP, int DB>
__device__ __forceinline__ void add_odd(const uint8_t* vt, int row0, int n, int key0, int last, int h, f16v (&acc)[DB]) {
#pragma unroll 1
  for (int j = 0; j < n; ++j) {
    if (key0 + j > last) continue;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const u2 w = *(const u2*)(vt + tile_off<DP>(row0 + j, 4 * d + g) + 8 * h);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[d][4 * g + i] += odd_part((w[i >> 1] >> (16 * (i & 1))) & 0xFFFFu);
      }
  }
}
template <int TK, int DP>
__device__ __forceinline__ void remove_odd(uint8_t* vt) {
  __syncthreads();
  for (int i = threadIdx.x; i < TK * DP / 8; i += 256) ((h8*)vt)[i] = finite_part(((const h8*)vt)[i]);
  __syncthreads();
}

// Many queries: 128 columns, 32 a wave; tiles of 64 keys, two blocks of 32, that the
// waves share. While the exponentials of key block b are taken, the scores of block
// b + 1 are formed and the probabilities of block b - 1 multiplied with v: a block's
// work is laid out in slices of two matrix instructions with the vector ones that
// fit under them, operands read AHEAD slices before. (A SIMD does not run one wave's
// exponentials under another's products by itself: in a probe the two took the sum
// of their times, 692 ns for 245 and 466, while 16 products with an exponential and
// three multiply-adds each, in one wave, took the products' 237.) k and v have two
// LDS buffers each, with one barrier a tile, in its middle: the first block is the
// last to use the older buffers.
// 4 x 4096 causal tokens, 32 heads of 128: 603 to 663 us on several cards, 830 to 910
// TFLOP/s, the matrix cores busy for 49 % of it. The card's power lowers its clock (one
// card took 634 us, and 472 with zeros for inputs); before results were stored by rows
// it was 650, and 820 with 64 queries a wave.
// K16, V16: whether k and v are F16 (and go straight into LDS) or have 8 bits.
template <int DP, bool K16, bool V16>
__global__ __launch_bounds__(256, 2) void attn_fwd_kernel(AttnParams p, int tiles) {
  constexpr int TK = 64, KS = DP / 16, DB = DP / 32, BUF = TK * DP * 2;
  constexpr int AHEAD = K16 && V16 ? 2 : 1;  // (the registers of staged tiles leave room for one)
  __shared__ __align__(16) uint8_t lds[4 * BUF];
  __shared__ int odd;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), h = lane >> 5;
  const Place at = attn_place(p, (int64_t)tiles * p.splits);
  const int split = (int)(at.rest % p.splits);
  // (the last columns see the most keys where the mask is causal: they go first)
  const int tile = tiles - 1 - (int)(at.rest / p.splits);
  const Seq sq = load_seq(p, at.b);
  const int64_t ncols = (int64_t)sq.lq * p.G, col0 = (int64_t)tile * 128;
  if (p.group0 + blockIdx.x == 0 && threadIdx.x == 0) *p.out_scale = pow2_float(clamp_e8m0(pow2_exponent(p.s_v)));
  if (col0 >= ncols) return;
  const int last0 = p.causal ? min((int)(col0 / p.G) + sq.behind, sq.lk - 1) : sq.lk - 1;  // of the first column
  const Query q = query_at(p, sq, at.hk, col0 + 32 * wave + (lane & 31), ncols);
  h8 qf[KS];
  load_row_operands(p.q_fmt, p.q, q.row * p.ldq + (int64_t)q.head * p.D, h, p.D, q.live, qf);
  int begin, end;
  key_range(p, sq, min(col0 + 127, ncols - 1), split, TK, begin, end);

  const float c1 = score_factor(p);
  float m = neg_inf(), l = 0.0f;
  f16v acc[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) acc[d] = f16v{};

  uint8_t* const kb = lds;
  uint8_t* const vb = lds + 2 * BUF;
  Tile<K16, TK, DP> lk;
  Tile<V16, TK, DP> lv;
  lk.init(p.k, sq.k0 * p.ldk + (int64_t)at.hk * p.D, p.ldk, p.D, p.k_fmt);
  lv.init(p.v, sq.k0 * p.ldv + (int64_t)at.hk * p.D, p.ldv, p.D, p.v_fmt);
  auto arrive = [&](uint8_t* kt, uint8_t* vt) {
    lk.arrive(kt);
    lv.arrive(vt);
    __syncthreads();
  };
  if (threadIdx.x == 0) odd = -1;
  f16v sa = {}, sb = {};
  h8 pa[2] = {}, pb[2] = {};  // probabilities of the last even and odd block
  if (begin < end) {
    lk.seek(begin);
    lv.seek(begin);
    lk.begin(end - begin, kb, wave);
#pragma unroll
    for (int i = 0; i < KS / 2; ++i) lk.issue(i);
    for (int i = threadIdx.x; i < BUF / 16; i += 256) ((u4*)(vb + BUF))[i] = u4{0u, 0u, 0u, 0u};  // (the block before the first)
    lk.arrive(kb);
    __syncthreads();
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) sa = mfma(row_operand<DP>(kb, 0, ks, lane), qf[ks], sa);
    lk.begin(end - begin - TK, kb + BUF, wave);
    lv.begin(end - begin, vb, wave);
#pragma unroll
    for (int i = 0; i < KS / 2; ++i) {
      lk.issue(i);
      lv.issue(i);
    }
  }
  settle_loads();

  // One block: its keys key0 ... with scores s, whose probabilities go to pn; the
  // next block's scores (rows kn of k) to sn, and the last block's probabilities pl
  // times its v (rows vl).
  auto block = [&](int key0, f16v& s, h8 (&pn)[2], f16v& sn, const uint8_t* kn, const h8 (&pl)[2], const uint8_t* vl, auto&& also) {
    if (key0 + 31 > last0) mask_scores(s, key0, h, q.last);
    const float off = kRunLog2 - (m == neg_inf() ? 0.0f : m);
    float lb = 0.0f, top = s[0];
    h8 kf[AHEAD + 1], vf[AHEAD + 1];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      kf[i] = row_operand<DP>(kn, 0, i, lane);
      vf[i] = col_operand<DP>(vl, 16 * (i / DB), i % DB, lane);
    }
    f16v sc = {};
    slice_end();
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      if (i + AHEAD < KS) {
        const int x = i + AHEAD;
        kf[x % (AHEAD + 1)] = row_operand<DP>(kn, 0, x, lane);
        vf[x % (AHEAD + 1)] = col_operand<DP>(vl, 16 * (x / DB), x % DB, lane);
      }
      also(i);
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        if (y == 0) sc = mfma(kf[i % (AHEAD + 1)], qf[i], sc);
        else acc[i % DB] = mfma(vf[i % (AHEAD + 1)], pl[i / DB], acc[i % DB]);
#pragma unroll
        for (int e = 8 / KS * (2 * i + y); e < 8 / KS * (2 * i + y + 1); ++e) {
          const float x = __builtin_amdgcn_exp2f(fmaf(s[e], c1, off));
          top = fmaxf(top, s[e]);  // (fmaxf skips NaN)
          lb += x;
          pn[e >> 3][e & 7] = (_Float16)x;
        }
        held(lb);
        slice_end();
      }
    }
    // The running maximum is moved only when a score is past it by more than
    // kSlack: with what had been added relative to the old one the block's
    // probabilities are then taken again.
    held(pn[0]);
    held(pn[1]);
    sn = sc;
    top = fmaxf(top, other_half(top, h)) * c1;
    if (__any(top > m + kSlack)) {
      const float now = fmaxf(m, top);
      const float f = m == neg_inf() ? 1.0f : __builtin_amdgcn_exp2f(m - now);  // (so far nothing but infinities may have been added)
      m = now;
      l *= f;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[d][r] *= f;
      const float o = kRunLog2 - (m == neg_inf() ? 0.0f : m);
      lb = 0.0f;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float x = __builtin_amdgcn_exp2f(fmaf(s[e], c1, o));
        lb += x;
        pn[e >> 3][e & 7] = (_Float16)x;
      }
    }
    l += lb;
  };
  int n = 0;  // the buffers of tile t
#pragma unroll 1
  for (int t = begin; t < end; t += TK, n ^= 1) {
    uint8_t* const kt = kb + n * BUF;
    uint8_t* const ko = kb + (n ^ 1) * BUF;
    uint8_t* const vt = vb + n * BUF;
    uint8_t* const vo = vb + (n ^ 1) * BUF;
    block(t, sa, pa, sb, kt + BUF / 2, pb, vo + BUF / 2, [](int) {});
    arrive(ko, vt);
    if (t + TK - 1 > last0) {  // some pair of the workgroup is masked
      mark_not_finite<TK, DP>(vt, &odd, t);
      __syncthreads();
      if (__builtin_amdgcn_readfirstlane(odd) == t) {
        add_odd<DP>(vt, 0, TK, t, q.last, h, acc);
        remove_odd<TK, DP>(vt);
      }
    }
    lk.begin(end - t - 2 * TK, kt, wave);
    lv.begin(end - t - TK, vo, wave);
    block(t + 32, sb, pb, sa, ko, pa, vt, [&](int i) {
      if (i < KS / 2) lk.issue(i);
      else lv.issue(i - KS / 2);
    });
  }
  if (begin < end) {  // the last block's product
    const uint8_t* const vl = vb + (n ^ 1) * BUF + BUF / 2;
#pragma unroll
    for (int i = 0; i < KS; ++i)
      acc[i % DB] = mfma(col_operand<DP>(vl, 16 * (i / DB), i % DB, lane), pb[i / DB], acc[i % DB]);
    wait_loads();  // (none may reach LDS after the workgroup has ended)
  }
  l += other_half(l, h);
  if (q.live && h == 0) store_row(p, q, m, l, split);
  const int64_t wave0 = col0 + 32 * wave;
  const bool part = p.splits > 1;
  __syncthreads();  // (the tiles have been read)
  store_rows<DP>(lds + wave * (32 * DP * 4), acc, part ? 1.0f : (l == 0.0f ? 0.0f : 1.0f / l), lane, (int)min((int64_t)32, ncols - wave0),
                 p.D, part ? p.part_o : nullptr, p.out, p.out_fmt, 0, p.sat != 0, [&](int r, int64_t& e32, int64_t& x) {
                   const int i = (int)(wave0 + r) / p.G, hd = at.hk * p.G + (int)(wave0 + r) - i * p.G;
                   e32 = ((split * p.rows_q + sq.q0 + i) * p.H + hd) * (int64_t)p.D;
                   x = (sq.q0 + i) * p.ldo + (int64_t)hd * p.D;
                 });
}

// Few queries: 32 columns, which each wave holds; every fourth block of 32 keys is a
// wave's, in an LDS tile of its own, so that no wave waits for another before the
// end, where the four are joined. (With tiles that the workgroup loaded together the
// barriers left memory idle: 32 single tokens over up to 4096 E4M3 keys of 8 heads took
// 82 us against 50, one over 131072 F16 keys 125 against 117, 4.6 TB/s.)
// K16, V16: whether k and v are F16 or have 8 bits.
template <int DP, bool K16, bool V16>
__global__ __launch_bounds__(256, 2) void attn_few_kernel(AttnParams p, int tiles) {
  // (F16 tiles go straight into LDS and have two buffers, 8-bit ones one: the next
  // tile's codes wait in registers)
  constexpr int TK = 128, KS = DP / 16, DB = DP / 32, BUF = 32 * DP * 2, NK = K16 ? 2 : 1, NV = V16 ? 2 : 1;
  __shared__ __align__(16) uint8_t lds[4 * (NK + NV) * BUF];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), h = lane >> 5;
  uint8_t* const kb = lds + wave * (NK + NV) * BUF;
  uint8_t* const vb = kb + NK * BUF;
  const Place at = attn_place(p, (int64_t)tiles * p.splits);
  const int split = (int)(at.rest % p.splits);
  const int tile = tiles - 1 - (int)(at.rest / p.splits);
  const Seq sq = load_seq(p, at.b);
  const int64_t ncols = (int64_t)sq.lq * p.G, col0 = (int64_t)tile * 32;
  if (p.group0 + blockIdx.x == 0 && threadIdx.x == 0) *p.out_scale = pow2_float(clamp_e8m0(pow2_exponent(p.s_v)));
  if (col0 >= ncols) return;
  const Query q = query_at(p, sq, at.hk, col0 + (lane & 31), ncols);
  int begin, end;
  key_range(p, sq, min(col0 + 31, ncols - 1), split, TK, begin, end);
  typename std::conditional<K16, WaveTile<DP>, StagedTile<32, DP, 64>>::type lk;
  typename std::conditional<V16, WaveTile<DP>, StagedTile<32, DP, 64>>::type lv;
  lk.init(p.k, sq.k0 * p.ldk + (int64_t)at.hk * p.D, p.ldk, p.D, p.k_fmt);
  lv.init(p.v, sq.k0 * p.ldv + (int64_t)at.hk * p.D, p.ldv, p.D, p.v_fmt);
  const int key0 = begin + 32 * wave;
  lk.skip(key0);
  lv.skip(key0);
  lk.begin(end - key0, kb, 0);
  lv.begin(end - key0, vb, 0);
  h8 qf[KS];
  load_row_operands(p.q_fmt, p.q, q.row * p.ldq + (int64_t)q.head * p.D, h, p.D, q.live, qf);
  const float c1 = score_factor(p);
  float m = neg_inf(), l = 0.0f;
  f16v acc[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) acc[d] = f16v{};

#pragma unroll 1
  for (int t = key0, n = 0; t < end; t += TK, n ^= 1) {
    uint8_t* const kt = kb + (K16 ? n * BUF : 0);
    uint8_t* const vt = vb + (V16 ? n * BUF : 0);
    wave_sync();  // (the block before has been read)
    lk.arrive(kt);
    lv.arrive(vt);
    wave_sync();
    lk.skip(3 * 32);
    lv.skip(3 * 32);
    lk.begin(end - t - TK, kb + (K16 ? (n ^ 1) * BUF : 0), 0);
    lv.begin(end - t - TK, vb + (V16 ? (n ^ 1) * BUF : 0), 0);
    const bool masked = __any(t + 31 > q.last);
    if (masked) {
      bool odd = false;
      for (int i = lane; i < 32 * DP / 8; i += 64) odd |= not_finite(((const h8*)vt)[i]);
      if (__any(odd)) {
        add_odd<DP>(vt, 0, 32, t, q.last, h, acc);
        wave_sync();
        for (int i = lane; i < 32 * DP / 8; i += 64) ((h8*)vt)[i] = finite_part(((const h8*)vt)[i]);
        wave_sync();
      }
    }
    f16v s = {};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) s = mfma(row_operand<DP>(kt, 0, ks, lane), qf[ks], s);
    if (masked) mask_scores(s, t, h, q.last);
    run_max(block_top(s), c1, h, m, l, acc);
    const float off = kRunLog2 - (m == neg_inf() ? 0.0f : m);
    float pr[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      pr[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c1, off));
      l += pr[r];
    }
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const h8 pf = to_operand(pr, g);
#pragma unroll
      for (int d = 0; d < DB; ++d) acc[d] = mfma(col_operand<DP>(vt, 16 * g, d, lane), pf, acc[d]);
    }
  }
  wait_loads();
  __syncthreads();
  l += other_half(l, h);

  // Join the four waves: maxima and sums first, then the scaled results, of which
  // wave w adds block w.
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
  if (wave < DB && q.live) {
    f16v o;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      float a = part[(wave * 16 + r) * 64 + lane];
#pragma unroll
      for (int w = 1; w < 4; ++w) a += part[((w * DB + wave) * 16 + r) * 64 + lane];
      o[r] = a;
    }
    store_result(p, o, q, wave, h, sum, split);
    if (wave == 0 && h == 0) store_row(p, q, top, sum, split);
  }
}

// Joins the splits of a query, a query a workgroup: eight groups of 32 lanes take
// every eighth split each, four columns a lane, and are added in order. (32 heads of 64
// splits: 7 us; a thread a column that walks the splits took 42.)
__global__ __launch_bounds__(256) void attn_join_kernel(AttnParams p) {
  __shared__ float4 part[8][32];
  __shared__ float sums[8];
  const int lane = threadIdx.x & 31, group = threadIdx.x >> 5;
  const Place at = attn_place(p, gridDim.x / (p.batch * p.Hkv));
  const Seq sq = load_seq(p, at.b);
  const int64_t col = at.rest;
  if (col >= (int64_t)sq.lq * p.G) return;
  const int pos = (int)(col / p.G), head = at.hk * p.G + (int)(col - (int64_t)pos * p.G);
  const int64_t row = sq.q0 + pos, first = row * p.H + head, step = p.rows_q * p.H;
  float m = neg_inf();
  for (int s = lane; s < p.splits; s += 32) m = fmaxf(m, p.part_ml[first + s * step].x);
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 32));
  float l = 0.0f, y[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s = group; s < p.splits; s += 8) {
    const float2 ml = p.part_ml[first + s * step];
    if (ml.y == 0.0f) continue;  // (nothing admitted)
    const float f = ml.x == neg_inf() ? 1.0f : __builtin_amdgcn_exp2f(ml.x - m);
    l += ml.y * f;
    if (4 * lane < p.D) {
      const float4 o = *(const float4*)(p.part_o + (first + s * step) * p.D + 4 * lane);
      y[0] += o.x * f;
      y[1] += o.y * f;
      y[2] += o.z * f;
      y[3] += o.w * f;
    }
  }
  part[group][lane] = make_float4(y[0], y[1], y[2], y[3]);
  if (lane == 0) sums[group] = l;
  __syncthreads();
  if (group != 0) return;
#pragma unroll
  for (int g = 1; g < 8; ++g) {
    const float4 o = part[g][lane];
    y[0] += o.x;
    y[1] += o.y;
    y[2] += o.z;
    y[3] += o.w;
    l += sums[g];
  }
  if (4 * lane < p.D) {
    const float inv = 1.0f / l;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = l == 0.0f ? 0.0f : y[i] * inv;
    store4_any(p.out_fmt, p.out, row * p.ldo + (int64_t)head * p.D + 4 * lane, y, 0, p.sat != 0);
  }
  if (p.lse && lane == 0) p.lse[(int64_t)head * p.rows_q + row] = log_sum(m, l);
}

__global__ void attn_scale_kernel(AttnParams p) {
  if (threadIdx.x == 0) *p.out_scale = pow2_float(clamp_e8m0(pow2_exponent(p.s_v)));
}

// 512 workgroups (two on each of the 256 CUs) fill the device. Both limits of the rule
// lie where neither side is better throughout (us, a captured call's kernels).
// Columns: the few-query kernel reads the keys once for each 32, the wide one has more
// products in flight. Few against wide: 40 columns over 8192 F16 keys of 4 heads 15.4,
// 17.6; 32 sequences of 40 over 4096 F16 keys of 8 heads 129, 124, over E4M3 keys 65, 93;
// 64 columns over 8192 keys of 8 heads 31, 23; 64 prompts of 48 tokens 26, 15.
// Keys of a split: without a split, from 256 keys on, from 128 on: 513 keys of 16 heads of
// 64 9.3, 9.9, 9.4; 1024 keys 10.6, 9.4, 9.0; 32 heads on 8 of 128, 2048 keys 22.5, 13.7,
// 12.7; 8192 keys 62.7, 17.2, 25.5.
AttnPlan attention_plan(int64_t batch, int Hkv, int G, int64_t max_q, int64_t max_k) {
  AttnPlan r;
  const int64_t cols = max_q * G;
  r.cols = cols <= 32 ? 32 : 128;
  const int64_t groups = batch * Hkv * ((cols + r.cols - 1) / r.cols);
  int64_t s = groups > 0 ? 512 / groups : 1;
  if (s > max_k / 256) s = max_k / 256;
  if (s > 64) s = 64;
  r.splits = s < 2 ? 1 : (int)s;
  return r;
}

template <int DP>
static hipError_t launch(const AttnParams& p, const AttnPlan& plan, hipStream_t s) {
  const int64_t cols = p.max_q * p.G;
  const int tiles = (int)((cols + plan.cols - 1) / plan.cols);
  const int64_t g = p.batch * p.Hkv * tiles * plan.splits;
  const bool k16 = p.k_fmt == kF16, v16 = p.v_fmt == kF16;
  if (plan.cols == 32) {
    if (k16 && v16) return launch_groups(attn_few_kernel<DP, true, true>, g, 1, s, p, tiles);
    if (k16) return launch_groups(attn_few_kernel<DP, true, false>, g, 1, s, p, tiles);
    if (v16) return launch_groups(attn_few_kernel<DP, false, true>, g, 1, s, p, tiles);
    return launch_groups(attn_few_kernel<DP, false, false>, g, 1, s, p, tiles);
  }
  if (k16 && v16) return launch_groups(attn_fwd_kernel<DP, true, true>, g, 1, s, p, tiles);
  if (k16) return launch_groups(attn_fwd_kernel<DP, true, false>, g, 1, s, p, tiles);
  if (v16) return launch_groups(attn_fwd_kernel<DP, false, true>, g, 1, s, p, tiles);
  return launch_groups(attn_fwd_kernel<DP, false, false>, g, 1, s, p, tiles);
}

hipError_t launch_attention_fwd(const AttnParams& p, const AttnPlan& plan, hipStream_t s) {
  if (p.rows_q == 0 || p.batch == 0 || p.max_q == 0) return launch_groups(attn_scale_kernel, 1, 1, s, p);
  const hipError_t e = p.D <= 64 ? launch<64>(p, plan, s) : launch<128>(p, plan, s);
  if (e != hipSuccess || plan.splits < 2) return e;
  // (keys are split for at most 256 tiles of at most 128 columns: one launch)
  return launch_groups(attn_join_kernel, p.batch * p.Hkv * p.max_q * p.G, 1, s, p);
}

}  // namespace scalify
