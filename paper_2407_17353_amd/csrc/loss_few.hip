// The losses for few rows (scored answers, single tokens, short batches): at most 128 of
// them, against the whole output matrix.
//
// Bound: the bytes of w, read once for the logits and once for dx, as they are stored
// (8-bit values become F16 in registers), and those of dw. Up to 16 rows, a workgroup takes
// 64 rows of w (tokens) and its four waves share the columns, 128 bytes of each row at a
// time in turn (512 contiguous bytes together); x comes from the L2 caches, where every
// workgroup finds it, and the waves' sums meet in LDS in a fixed order. With more rows
// that x would be several bytes for each of w (48 rows of 4096 columns: 79 us, now 35, with w's bytes
// alone 27): the waves then take 16 tokens each and go through x together, in LDS, the
// columns of w and x loaded three chunks ahead. Measured (131 MB of w: 27 us at the rate of a
// large copy): logits of 16 rows, 2048 columns in F16, 26 us; 48 rows, 4096 in 8 bits, 32, of 128
// rows 56 (LDS reads and the products, 25 us each, meet the bytes). So with w in the last-level
// cache from the call before; with another w of six in turn, the calls take 39 us for 30 (16
// rows) and 44 for 34 (48).
// The forward goes over every row, those that do not count too (their results are 0, and
// nothing of them reaches another's); the backward over those that count. Either picks its
// kernels by the number of rows, all that the host knows.
#include "attention_dev.h"
#include "kernels.h"
#include "loss_dev.h"

#include <algorithm>
#include <type_traits>

namespace scalify {

typedef float f4 __attribute__((ext_vector_type(4)));

constexpr int FEW_TOKENS = 64;

// k of a lane in a chunk of 128 bytes of a row of w.
template <int FW>
constexpr int few_k() {
  return FW == kF16 ? 16 : 32;
}

// Eight F16 values, those from column `left` on 0.
__device__ __forceinline__ u4 mask8(u4 v, int left) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] &= (2 * i < left ? 0xFFFFu : 0u) | (2 * i + 1 < left ? 0xFFFF0000u : 0u);
  return v;
}

// Eight of the 16-byte groups of a chunk of w as an operand.
template <int FW>
__device__ __forceinline__ u4 weights8(const u4 (&c)[2], int i) {
  if constexpr (FW == kF16) {
    return c[i];
  } else {
    const u4 v = c[i >> 1];
    return to_f16x8(FW, i & 1 ? u4{v[2], v[3], 0u, 0u} : u4{v[0], v[1], 0u, 0u});
  }
}

// What a workgroup does with its logits' sums z[part][token][place ^ permutation]: a thread
// has a place and consecutive tokens.
__device__ __forceinline__ int few_at(int token, int place) { return place ^ (4 * ((token >> 2) & 3)); }

template <int PLACES, int PARTS, bool BACK>
__device__ __forceinline__ void finish_few(const LossParams& p, const float* z, int t0, int R) {
  constexpr int SH = 256 / PLACES, PER = FEW_TOKENS / SH;
  const int place = threadIdx.x / SH, share = threadIdx.x % SH;
  auto sum_at = [&](int t, int pl) {
    float s = z[t * PLACES + few_at(t, pl)];
    if constexpr (PARTS == 4) {
      const int o = t * PLACES + few_at(t, pl), n = FEW_TOKENS * PLACES;
      s = (s + z[o + n]) + (z[o + 2 * n] + z[o + 3 * n]);
    }
    return s;
  };
  const bool in = place < R;
  if constexpr (BACK) {
    if (!in) return;
    const float f = p.factor[place], l = p.lse2[place], c = p.coef[place];
    const int label = p.labels ? p.label[place] - t0 : -1;
    _Float16* to = (_Float16*)p.dz + (int64_t)place * p.ldz + t0 + share * PER;  // (a pitch holds whole groups of 64)
#pragma unroll
    for (int b = 0; b < PER / 4; ++b) {
      _Float16 y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int t = share * PER + 4 * b + i;
        float v = c * __builtin_amdgcn_exp2f(held_log(__builtin_fmaf(sum_at(t, place), f, -l), l));
        if (t == label) v -= c;
        y[i] = (_Float16)(t0 + t < p.V ? v : 0.f);
      }
      typedef _Float16 h4 __attribute__((ext_vector_type(4)));
      *(h4*)(to + 4 * b) = h4{y[0], y[1], y[2], y[3]};
    }
    return;
  }
  float v[PER], top = -__builtin_inff();
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int t = share * PER + i;
    v[i] = t0 + t < p.V ? sum_at(t, place) : -__builtin_inff();
    top = fmaxf(top, v[i]);
  }
#pragma unroll
  for (int o = 1; o < SH; o <<= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
  const float f = in ? logit_factor(p, place) : 0.f;
  const float m2 = top == -__builtin_inff() || top != top ? 0.f : top * f;
  const bool large = is_large(m2);
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < PER; ++i) sum += __builtin_amdgcn_exp2f(large ? (v[i] - top) * f : __builtin_fmaf(v[i], f, -m2));
#pragma unroll
  for (int o = 1; o < SH; o <<= 1) sum += __shfl_xor(sum, o, 64);
  if (in && share == 0) p.stats[(int64_t)place * gridDim.x + blockIdx.x] = float2{sum == 0.f ? -__builtin_inff() : m2, sum};
  if (p.labels) {
    if (in) {
      const int64_t d = p.labels[place] - t0;
      if (d >= share * PER && d < (share + 1) * PER && d + t0 < p.V) p.picked2[place] = sum_at((int)d, place) * f;
    }
  } else {
    // (the whole list, whose numbers are in the L2 caches: it costs by its length. 128 rows against
    // 32000 x 2048 in 8 bits 38 us with 8 entries a row, 45 with 64, 76 with 256)
    for (int e = threadIdx.x; e < p.R * p.top; e += 256) {
      const int64_t d = p.index[e] - t0;
      if (d >= 0 && d < FEW_TOKENS && d + t0 < p.V) p.picked[e] = sum_at((int)d, e / p.top) * (logit_factor(p, e / p.top) * kLn2);
    }
  }
}

// At most 16 rows. BACK: dz of the places (rows that count, as F16 in xc), else the rows'
// statistics.
template <int FW, bool X16, bool BACK>
__global__ __launch_bounds__(256) void loss_few_kernel(LossParams p) {
  constexpr int MT = FEW_TOKENS / 16, KL = few_k<FW>(), KC = 4 * KL, G8 = KL / 8, XG = X16 ? G8 : G8 / 2;
  __shared__ float z[4][FEW_TOKENS][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int t0 = blockIdx.x * FEW_TOKENS, D = p.D;
  constexpr int esz = FW == kF16 ? 2 : 1;
  const int R = BACK ? (int)p.hdr[LOSS_COUNT] : p.R;
  if (BACK && R == 0) return;
  const uint8_t* wr[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) wr[m] = (const uint8_t*)p.w + (int64_t)min(t0 + 16 * m + r, p.V - 1) * p.ldw * esz;
  const uint8_t* const xr = (const uint8_t*)(BACK ? p.xc : p.x) + (int64_t)min(r, R - 1) * (BACK ? p.ldxc : p.ldx) * (X16 ? 2 : 1);
  f4 acc[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) acc[m] = f4{0.f, 0.f, 0.f, 0.f};

  // A lane's part of the chunk at k0: k = k0 + KL g ... Groups that start past the
  // row's end are 0 and not read (a pitch holds whole groups of 16 bytes).
  u4 wc[2][MT][2], xc[2][XG];
  auto load = [&](int k0, u4 (&w)[MT][2], u4 (&x)[XG]) {
    const int k = k0 + KL * g;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int at = k + KL / 2 * h;
#pragma unroll
      for (int m = 0; m < MT; ++m) w[m][h] = at < D ? *(const u4*)(wr[m] + (int64_t)at * esz) : u4{0u, 0u, 0u, 0u};
    }
#pragma unroll
    for (int i = 0; i < XG; ++i) {
      const int at = k + KL / XG * i;
      x[i] = at < D ? *(const u4*)(xr + (X16 ? 2 : 1) * at) : u4{0u, 0u, 0u, 0u};
    }
  };
  auto multiply = [&](int k0, const u4 (&w)[MT][2], const u4 (&x)[XG]) {
    const int left = D - (k0 + KL * g);
    const bool tail = k0 + KC > D;
#pragma unroll
    for (int i = 0; i < G8; ++i) {
      u4 v;
      if constexpr (X16) {
        v = x[i];
      } else {
        const u4 c = x[i / 2];
        v = to_f16x8(p.x_fmt, i & 1 ? u4{c[2], c[3], 0u, 0u} : u4{c[0], c[1], 0u, 0u});
      }
      if (tail) v = mask8(v, left - 8 * i);
      const h8 b = __builtin_bit_cast(h8, v);
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        u4 a = weights8<FW>(w[m], i);
        if (tail) a = mask8(a, left - 8 * i);
        acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), b, acc[m], 0, 0, 0);
      }
    }
  };
  int k0 = wave * KC;
  load(k0, wc[0], xc[0]);
  while (k0 < D) {
    load(k0 + 4 * KC, wc[1], xc[1]);
    multiply(k0, wc[0], xc[0]);
    k0 += 4 * KC;
    if (k0 >= D) break;
    load(k0 + 4 * KC, wc[0], xc[0]);
    multiply(k0, wc[1], xc[1]);
    k0 += 4 * KC;
  }
  // a lane holds tokens 16 m + 4 g + i of place r
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = 16 * m + 4 * g + i;
      z[wave][t][few_at(t, r)] = acc[m][i];
    }
  __syncthreads();
  finish_few<16, 4, BACK>(p, &z[0][0][0], t0, R);
}

// Up to 16 NP rows, their columns in LDS. Products go by groups of 16 rows, as do LDS reads: NP
// 3 and 6 beside 2, 4 and 8 (4096 columns in 8 bits, 48 rows: 41 us as 64, 35 as 48; 96 rows 62
// and 52). F16's chunks of 64 columns need an even NP, a whole number of loads a thread; 5 and 7,
// for 80 and 112 rows of 8 bits, have not been tried. (X16 is a template's so that 8-bit rows of x wait in
// half the registers: read in either form by a branch, 128 rows against 32000 x 4096 in E4M3
// took 137 us, now 60.)
template <int FW, int NP, bool X16, bool BACK>
__global__ __launch_bounds__(256) void loss_rows_kernel(LossParams p) {
  constexpr int KL = few_k<FW>(), KC = 4 * KL, G8 = KL / 8, PLACES = 16 * NP, ROW = 2 * KC, CH = ROW / 16;
  constexpr int NG = PLACES * CH / 256;  // groups of eight of a chunk of x that a thread loads
  constexpr int BUF = PLACES * ROW;
  constexpr int ZP = NP <= 2 ? 32 : (NP <= 4 ? 64 : 128);  // places of a token's logits (those past PLACES hold anything)
  constexpr int BYTES = 2 * BUF > FEW_TOKENS * ZP * 4 ? 2 * BUF : FEW_TOKENS * ZP * 4;
  static_assert(PLACES * CH % 256 == 0, "whole groups a thread");
  __shared__ __attribute__((aligned(16))) uint8_t smem[BYTES];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int t0 = blockIdx.x * FEW_TOKENS, D = p.D;
  constexpr int esz = FW == kF16 ? 2 : 1;
  const int R = BACK ? (int)p.hdr[LOSS_COUNT] : p.R;
  if (BACK && R == 0) return;
  constexpr int xsz = X16 ? 2 : 1;
  typedef std::conditional_t<X16, u4, u2> Group;  // eight columns of x
  const uint8_t* const x0 = (const uint8_t*)(BACK ? p.xc : p.x);
  const int64_t xpitch = (BACK ? p.ldxc : p.ldx) * xsz;
  const uint8_t* const wr = (const uint8_t*)p.w + (int64_t)min(t0 + 16 * wave + r, p.V - 1) * p.ldw * esz;
  // group j of a thread: 16-byte place c of a place's row in LDS, permuted by the place
  const uint8_t* xr[NG];
  int xk[NG], xl[NG];
#pragma unroll
  for (int j = 0; j < NG; ++j) {
    const int q = (int)threadIdx.x + 256 * j, place = q / CH, c = q % CH;
    xr[j] = x0 + (int64_t)min(place, R - 1) * xpitch;
    xk[j] = 8 * c;
    xl[j] = place * ROW + ((c ^ (CH == 8 ? (place & 7) ^ ((place >> 3) & 1) : place & 15)) << 4);
  }
  f4 acc[NP];
#pragma unroll
  for (int n = 0; n < NP; ++n) acc[n] = f4{0.f, 0.f, 0.f, 0.f};
  u4 w[3][2];
  Group x[3][NG];
  auto load = [&](int k0, u4 (&wo)[2], Group (&xo)[NG]) {
#pragma unroll
    for (int j = 0; j < NG; ++j) {
      const int at = k0 + xk[j];
      xo[j] = at < D ? *(const Group*)(xr[j] + xsz * at) : Group{};
    }
    const int k = k0 + KL * g;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int at = k + KL / 2 * h;
      wo[h] = at < D ? *(const u4*)(wr + (int64_t)at * esz) : u4{0u, 0u, 0u, 0u};
    }
  };
  auto put = [&](int k0, uint8_t* lds, const Group (&xi)[NG]) {
#pragma unroll
    for (int j = 0; j < NG; ++j) {
      u4 v;
      if constexpr (X16) {
        v = xi[j];
      } else {
        const u4 c = u4{xi[j][0], xi[j][1], 0u, 0u};
        v = p.x_fmt == kE4M3 ? to_f16x8(kE4M3, c) : to_f16x8(kE5M2, c);
      }
      if (k0 + KC > D) v = mask8(v, D - (k0 + xk[j]));
      *(u4*)(lds + xl[j]) = v;
    }
  };
  auto multiply = [&](int k0, const uint8_t* lds, const u4 (&wi)[2]) {
#pragma unroll
    for (int i = 0; i < G8; ++i) {
      u4 a = weights8<FW>(wi, i);
      if (k0 + KC > D) a = mask8(a, D - (k0 + KL * g + 8 * i));
      const int c = G8 * g + i;
#pragma unroll
      for (int n = 0; n < NP; ++n) {
        const int place = 16 * n + r;
        const h8 b = *(const h8*)(lds + place * ROW + ((c ^ (CH == 8 ? (place & 7) ^ ((place >> 3) & 1) : place & 15)) << 4));
        acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), b, acc[n], 0, 0, 0);
      }
    }
  };
#pragma unroll
  for (int j = 0; j < 3; ++j) load(j * KC, w[j], x[j]);
  // (a wave that stores into a buffer has passed the barrier that follows the last use of it)
  for (int k0 = 0; k0 < D; k0 += 6 * KC) {
#pragma unroll
    for (int j = 0; j < 6; ++j) {
      const int k = k0 + j * KC;
      if (k < D) {
        uint8_t* lds = smem + (j & 1) * BUF;
        put(k, lds, x[j % 3]);
        const u4 now[2] = {w[j % 3][0], w[j % 3][1]};
        load(k + 3 * KC, w[j % 3], x[j % 3]);
        __syncthreads();
        multiply(k, lds, now);
      }
    }
  }
  __syncthreads();
  float* z = (float*)smem;
#pragma unroll
  for (int n = 0; n < NP; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = 16 * wave + 4 * g + i;
      z[t * ZP + few_at(t, 16 * n + r)] = acc[n][i];
    }
  __syncthreads();
  finish_few<ZP, 1, BACK>(p, z, t0, R);
}

// ---- the gradients' products of few rows, from their dz

// dx: places x 128 columns, over a part of the vocabulary (blockIdx.y, `per` tokens), 64
// tokens' rows of w and their dz at a time through LDS. Bound: the bytes of w. The matrix
// instruction's operands: a lane has a column of w and the tokens in the order that the
// transposing read gives them, and a place's dz in the same order. 32000 x 2048 in F16: 22 us
// for 16 rows, 37 for 128; 32000 x 4096 in 8 bits, decoded on the way into LDS, 28 and 66.
template <bool W16, int NT>
__global__ __launch_bounds__(256) void loss_few_dx_kernel(LossParams p, int per) {
  __shared__ __attribute__((aligned(1024))) uint8_t tiles[2][64 * 256], grads[2][32 * NT * 128];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const int col0 = blockIdx.x * 128, cols = W16 ? (p.D + 7) & ~7 : (p.D + 15) & ~15;
  const int count = (int)p.hdr[LOSS_COUNT];
  const int first = blockIdx.y * per, end = min(p.V, first + per);
  if (count == 0) return;
  Tile<W16, 64, 128> tw;
  tw.init(p.w, col0, p.ldw, cols - col0, p.w_fmt);
  tw.seek(first);
  f16v acc[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[n][i] = 0.f;
  auto begin = [&](int t0, int at) {
    tw.begin(end - t0, tiles[at], wave);
#pragma unroll
    for (int i = 0; i < 4; ++i) tw.issue(i);
    // (dz's rows hold 0 past V, up to a whole tile)
    DirectTile<32 * NT, 64> td;
    td.init(p.dz, t0, p.ldz, 64, kF16);
    td.seek(0);
    td.begin(count, grads[at], wave);
#pragma unroll
    for (int i = 0; i < NT; ++i) td.issue(i);
  };
  auto arrive = [&](int at) {
    tw.arrive(tiles[at]);
    wait_loads();
    __syncthreads();
  };
  auto multiply = [&](int at) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const h8 a = col_operand<128>(tiles[at], 16 * k, wave, lane);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const int row = 32 * n + (lane & 31);
        const u2 lo = *(const u2*)(grads[at] + tile_off<64>(row, 2 * k) + 8 * h), hi = *(const u2*)(grads[at] + tile_off<64>(row, 2 * k + 1) + 8 * h);
        acc[n] = mfma(a, __builtin_bit_cast(h8, u4{lo[0], lo[1], hi[0], hi[1]}), acc[n]);
      }
    }
  };
  if (first < end) {
    begin(first, 0);
    arrive(0);
    int at = 0;
    for (int t0 = first; t0 < end; t0 += 64, at ^= 1) {
      const bool more = t0 + 64 < end;
      if (more) begin(t0 + 64, at ^ 1);
      multiply(at);
      if (more) arrive(at ^ 1);
    }
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int place = 32 * n + (lane & 31);
    if (place < count) {
      const float f = p.dx_factor[place];
      float* o = p.part + ((int64_t)blockIdx.y * p.R + place) * p.ldp;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int c = col0 + 32 * wave + 8 * g + 4 * h;
        if (c < p.ldp) *(float4*)(o + c) = make_float4(acc[n][4 * g] * f, acc[n][4 * g + 1] * f, acc[n][4 * g + 2] * f, acc[n][4 * g + 3] * f);
      }
    }
  }
}

template <int N>
__device__ __forceinline__ void wait_some() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// dw: 128 columns, whose x a workgroup keeps in registers, over a part of the vocabulary
// (blockIdx.y, `per` tokens), 64 tokens' dz at a time through LDS. Bound: the bytes of
// dw. A wave's 32 tokens x 64 columns go through its own LDS so that half a row (128 bytes of
// F16) is stored at once; they become codes before that (32000 x 4096 in F16, 48 rows: 56 us;
// fp32 through LDS and cast on the way out, 100). OF: the codes' format, or FORM_NONE, the
// statistic alone: the dynamic rescale goes over the products twice, which costs less than
// their bytes in between would (64 rows, 50021 x 2048 in 8 bits: the backward 185 us, was 233).
// 32000 x 2048 in F16: 24 us for one row (5.4 TB/s), 38 for 128.
template <int NT, int OF>
__global__ __launch_bounds__(256) void loss_few_dw_kernel(LossParams p, int per) {
  constexpr int ESZ = OF == kF16 ? 2 : 1, F8 = OF == kE4M3 ? kE4M3 : kE5M2;
  constexpr int PER = 16 / ESZ, LPR = 64 / PER;  // elements of a lane's store, lanes of a row
  constexpr int KS = 2 * NT;  // products of 16 places
  constexpr int ROW = 64 * ESZ, CH = ROW / 16;  // a token's bytes in a wave's LDS, and their chunks
  __shared__ __attribute__((aligned(1024))) uint8_t sd[3][32 * NT * 128], sx[8192 * NT > 8192 * ESZ ? 8192 * NT : 8192 * ESZ];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const int col0 = blockIdx.x * 128, count = (int)p.hdr[LOSS_COUNT], cols = (p.D + 7) & ~7;
  const int first = blockIdx.y * per, end = min(p.V, first + per);
  if (first >= end) return;
  const int base = base_of(p, true), unit = unit_of(p, true), shift = out_exponent(p, true, base, unit) - base - unit;
  const bool fast = shift >= kFastShiftMinSub && shift <= kFastShiftMax;
  const float scale = fast ? pow2_float(shift) : 1.0f, inv = fast ? pow2_float(-shift) : 1.0f;
  auto begin = [&](int t0, int at) {
    DirectTile<32 * NT, 64> td;
    td.init(p.dz, __builtin_amdgcn_readfirstlane(t0), p.ldz, 64, kF16);
    td.seek(0);
    td.begin(__builtin_amdgcn_readfirstlane(count), sd[__builtin_amdgcn_readfirstlane(at)], wave);
#pragma unroll
    for (int i = 0; i < NT; ++i) td.issue(i);
  };
  DirectTile<32 * NT, 128> tx;
  tx.init(p.xw ? p.xw : p.xc, col0, p.ldxc, cols - col0, kF16);
  tx.seek(0);
  tx.begin(count, sx, wave);
#pragma unroll
  for (int i = 0; i < 2 * NT; ++i) tx.issue(i);
  wait_loads();
  __syncthreads();
  const int tt = wave & 1, cc = wave >> 1;  // the wave's tokens and columns
  h8 a[2][KS];
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int k = 0; k < KS; ++k) a[c][k] = col_operand<128>(sx, 16 * k, 2 * cc + c, lane);
  settle_loads();
  __syncthreads();
  uint8_t* const out = sx + wave * 32 * ROW;  // [32 tokens][64 columns], the chunks of a row permuted by it
  float lmax = 0.f;
  // dz is loaded two steps ahead. Vector memory is done in order: behind a step's loads there
  // are the next step's, and the stores of two steps, which so need not be waited for.
  constexpr int STORES = OF == FORM_NONE ? 0 : 32 / PER;
  const bool stores = col0 + 64 * cc + 64 <= p.D;  // all of them, in every step but the last
  begin(first, 0);
  if (first + 64 < end) begin(first + 64, 1);
  int step = 0, at = 0;
  for (int t0 = first; t0 < end; t0 += 64, ++step, at = at == 2 ? 0 : at + 1) {
    if (!stores || t0 + 64 >= end)
      wait_loads();
    else if (step == 0)
      wait_some<NT>();
    else if (step == 1)
      wait_some<NT + STORES>();
    else
      wait_some<NT + 2 * STORES>();
    __syncthreads();
    if (t0 + 128 < end) begin(t0 + 128, at == 0 ? 2 : at - 1);
    f16v acc[2];
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[c][i] = 0.f;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const h8 b = col_operand<64>(sd[at], 16 * k, tt, lane);
#pragma unroll
      for (int c = 0; c < 2; ++c) acc[c] = mfma(a[c][k], b, acc[c]);
    }
    // (columns past D are 0, as x's are)
    if (OF == FORM_NONE || (p.mode != 1 && p.amax_out)) {
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) lmax = fmaxf(lmax, fabsf(acc[c][i]));
    }
    if constexpr (OF == FORM_NONE) continue;
    const int r = lane & 31;
    wave_sync();
    auto stage = [&](auto nan_tag) {
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int o = (32 * c + 8 * g + 4 * h) * ESZ;  // of the row's bytes
          uint8_t* to = out + r * ROW + (((o >> 4) ^ (r & (CH - 1))) << 4) + (o & 15);
          const float y[4] = {acc[c][4 * g], acc[c][4 * g + 1], acc[c][4 * g + 2], acc[c][4 * g + 3]};
          if constexpr (OF == kF16) {
            *(u2*)to = codes4_f16<decltype(nan_tag)::value>(y, inv, p.sat);
          } else {
            *(uint32_t*)to = codes4_fp8<F8, decltype(nan_tag)::value>(y, scale, p.sat);
          }
        }
    };
    if (!fast) {  // exact wherever the result is normal, below it 0 either way
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[c][i] = __builtin_amdgcn_ldexpf(acc[c][i], -shift);
    }
    float any = 0.f;  // (NaN if there is one, or two infinities)
#pragma unroll
    for (int i = 0; i < 16; ++i) any += acc[0][i] + acc[1][i];
    if (__builtin_expect(__ballot(any != any) != 0, 0))
      stage(std::true_type{});
    else
      stage(std::false_type{});
    wave_sync();
    const int q = lane % LPR, c = col0 + 64 * cc + PER * q, n = p.D - c;
#pragma unroll
    for (int j = 0; j < 32 / PER; ++j) {
      const int row = PER * j + lane / LPR, t = t0 + 32 * tt + row;
      if (t < end && n > 0) {
        const u4 w = *(const u4*)(out + row * ROW + ((q ^ (row & (CH - 1))) << 4));
        uint8_t* to = (uint8_t*)p.dw + ((int64_t)t * p.lddw + c) * ESZ;
        if (n >= PER) {
          *(u4*)to = w;
        } else {
#pragma unroll
          for (int i = 0; i < PER - 1; ++i)
            if (i < n) {
              if constexpr (ESZ == 2)
                ((uint16_t*)to)[i] = (uint16_t)(w[i / 2] >> (16 * (i % 2)));
              else if constexpr (ESZ == 1)
                to[i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
            }
        }
      }
    }
  }
  if (OF != FORM_NONE && (p.mode == 1 || !p.amax_out)) return;
  lmax = wave_max(lmax);
  __syncthreads();
  float* const most = (float*)sx;
  if (lane == 0) most[wave] = lmax;
  __syncthreads();
  if (threadIdx.x == 0) raise_amax(p.hdr + LOSS_AMAX_DW, fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])));
}

// ---- host

template <int FW, bool X16, bool BACK>
static hipError_t launch_tokens(const LossParams& p, int groups, hipStream_t s) {
  if (p.R <= 16) return launch_one(loss_few_kernel<FW, X16, BACK>, groups, 256, s, p);
  if (p.R <= 32) return launch_one(loss_rows_kernel<FW, 2, X16, BACK>, groups, 256, s, p);
  if constexpr (FW != kF16) {
    if (p.R <= 48) return launch_one(loss_rows_kernel<FW, 3, X16, BACK>, groups, 256, s, p);
  }
  if (p.R <= 64) return launch_one(loss_rows_kernel<FW, 4, X16, BACK>, groups, 256, s, p);
  if (p.R <= 96) return launch_one(loss_rows_kernel<FW, 6, X16, BACK>, groups, 256, s, p);
  return launch_one(loss_rows_kernel<FW, 8, X16, BACK>, groups, 256, s, p);
}

template <bool X16, bool BACK>
static hipError_t launch_logits(const LossParams& p, int groups, hipStream_t s) {
  if (p.w_fmt == kF16) return launch_tokens<kF16, X16, BACK>(p, groups, s);
  if (p.w_fmt == kE4M3) return launch_tokens<kE4M3, X16, BACK>(p, groups, s);
  return launch_tokens<kE5M2, X16, BACK>(p, groups, s);
}

int loss_few_groups(const LossParams& p) { return (p.V + FEW_TOKENS - 1) / FEW_TOKENS; }

hipError_t launch_loss_few(const LossParams& p, hipStream_t s) {
  const int groups = loss_few_groups(p);
  return p.x_fmt == kF16 ? launch_logits<true, false>(p, groups, s) : launch_logits<false, false>(p, groups, s);
}

hipError_t launch_loss_few_dz(const LossParams& p, hipStream_t s) {
  return launch_logits<true, true>(p, loss_few_groups(p), s);
}

// A workgroup 128 columns and a part of the vocabulary, of whole tiles of 64 tokens.
static hipError_t launch_parts(void (*kernel)(LossParams, int), const LossParams& p, int parts, hipStream_t s) {
  LossParams q = p;
  int per = ((p.V + parts - 1) / parts + 63) / 64 * 64;
  void* a[] = {&q, &per};
  const hipError_t e = hipLaunchKernel((const void*)kernel, dim3((unsigned)((p.D + 127) / 128), (unsigned)parts), dim3(256), a, 0, s);
  if (e != hipSuccess) (void)hipGetLastError();
  return e;
}

hipError_t launch_loss_few_grads(const LossParams& p, hipStream_t s) {
  const int nt = p.R <= 32 ? 1 : (p.R <= 64 ? 2 : 4);
  if (p.dx_scale) {
    const bool w16 = p.w_fmt == kF16;
    const hipError_t e = launch_parts(nt == 1   ? (w16 ? loss_few_dx_kernel<true, 1> : loss_few_dx_kernel<false, 1>)
                                      : nt == 2 ? (w16 ? loss_few_dx_kernel<true, 2> : loss_few_dx_kernel<false, 2>)
                                                : (w16 ? loss_few_dx_kernel<true, 4> : loss_few_dx_kernel<false, 4>),
                                      p, p.splits, s);
    if (e != hipSuccess) return e;
  }
  if (!p.dw_scale) return hipSuccess;
  // parts: 4 workgroups for each CU
  const int tiles = (p.D + 127) / 128;
  const int parts = std::max(1, std::min((p.V + 63) / 64, 4 * gemm4_grid(1 << 30) / tiles));
  auto launch = [&](auto form) {
    constexpr int OF = decltype(form)::value;
    return launch_parts(nt == 1 ? loss_few_dw_kernel<1, OF> : nt == 2 ? loss_few_dw_kernel<2, OF> : loss_few_dw_kernel<4, OF>, p, parts, s);
  };
  if (p.mode == 1) {
    const hipError_t e = launch(std::integral_constant<int, FORM_NONE>{});
    if (e != hipSuccess) return e;
  }
  if (p.dw_fmt == kF16) return launch(std::integral_constant<int, kF16>{});
  return p.dw_fmt == kE4M3 ? launch(std::integral_constant<int, kE4M3>{}) : launch(std::integral_constant<int, kE5M2>{});
}

}  // namespace scalify
