// Device helpers of the attention kernels: sequences, tiles of keys (or
// queries) in LDS, and the matrix operands read from them.
//
// All products run on the F16 matrix instruction (32 x 32 x 16, fp32 sums):
// every E4M3 and E5M2 value is an F16 value, so 8-bit operands are decoded
// exactly on their way into LDS.
//
// Operand order. The instruction's result gives a lane one column (lane & 31)
// and, of its half h = lane >> 5, rows 8 (r / 4) + 4 h + r % 4 in register r; its
// operands give a lane one row or column and the eight consecutive k of its half.
// A product whose k runs over another's rows therefore takes that result without
// any exchange between lanes, if the other operand's k are permuted alike: of 16
// rows, half 0 holds 0-3 and 8-11, half 1 holds 4-7 and 12-15. The transposing
// LDS read gives just that: each 16 lanes read four rows of 16 columns and every
// lane receives its column's four values, so two reads make an operand.
#pragma once
#include "attention.h"
#include "codec.h"
#include "ew_util.h"

#include <type_traits>

namespace scalify {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef unsigned int u2 __attribute__((ext_vector_type(2)));
#define ATTN_LDS __attribute__((address_space(3)))

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
// Probabilities are kept as 2^14 p (at most 2^14): in F16 the normal range then
// reaches down to p = 2^-28, where 2^-14, a uniform row over 16384 keys, would be
// its end.
constexpr float kProbLog2 = 14.0f;

__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }

// A sequence's rows. Device arrays are not checked by the host: whatever they
// hold, the rows stay inside the matrices.
struct Seq {
  int64_t q0, k0;
  int lq, lk, kext;  // queries (up to max_q), keys, key rows of the sequence (keys past lk are padding)
  int behind;        // a causal mask lets query i see the keys up to i + behind: lk less all of the sequence's queries
};

__device__ __forceinline__ int64_t clamp64(int64_t x, int64_t lo, int64_t hi) {
  return x < lo ? lo : (x > hi ? hi : x);
}

__device__ __forceinline__ Seq load_seq(const AttnParams& p, int64_t b) {
  Seq s;
  int64_t q1, k1;
  if (p.q_start) {
    s.q0 = clamp64(p.q_start[b], 0, p.rows_q);
    q1 = clamp64(p.q_start[b + 1], s.q0, p.rows_q);
  } else {
    const int64_t n = (uint32_t)p.rows_q / (uint32_t)p.batch;  // (both at most 2^30)
    s.q0 = b * n;
    q1 = s.q0 + n;
  }
  if (p.k_start) {
    s.k0 = clamp64(p.k_start[b], 0, p.rows_k);
    k1 = clamp64(p.k_start[b + 1], s.k0, p.rows_k);
  } else {
    const int64_t n = (uint32_t)p.rows_k / (uint32_t)p.batch;
    s.k0 = b * n;
    k1 = s.k0 + n;
  }
  const int64_t lq = q1 - s.q0;
  s.lq = (int)(lq < p.max_q ? lq : p.max_q);
  s.kext = (int)(k1 - s.k0);
  s.lk = p.k_len ? (int)clamp64(p.k_len[b], 0, s.kext) : s.kext;
  s.behind = s.lk - (int)lq;
  return s;
}

// Byte offset of 16-byte chunk c of a row in an LDS tile of DP columns. Chunks
// are permuted within a row so that neither reading the same chunk of
// consecutive rows (16 bytes a lane) nor four neighbouring chunks of four rows
// (the transposing read) meets a bank twice.
template <int DP>
__device__ __forceinline__ int tile_off(int row, int c) {
  const int f = DP == 128 ? (((row & 3) << 2) | ((row >> 2) & 3)) : ((((row >> 1) & 1) << 2) | ((row >> 2) & 3));
  return row * (DP * 2) + ((c ^ f) << 4);
}

__device__ __forceinline__ int fmt_bytes(int fmt) { return fmt == kF16 ? 2 : 1; }

// Eight codes of a format, as they were loaded (16 or 8 bytes), as F16.
__device__ __forceinline__ u4 to_f16x8(int fmt, u4 w) {
  if (fmt == kF16) return w;
  u4 r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    h2 lo, hi;
    if (fmt == kE4M3) {
      lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i], 1.0f, false);
      hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i], 1.0f, true);
    } else {
      lo = __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(w[i], 1.0f, false);
      hi = __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(w[i], 1.0f, true);
    }
    r[2 * i] = __builtin_bit_cast(uint32_t, lo);
    r[2 * i + 1] = __builtin_bit_cast(uint32_t, hi);
  }
  return r;
}

// Eight consecutive codes at element e of base, as F16.
__device__ __forceinline__ u4 load_f16x8(int fmt, const void* base, int64_t e) {
  if (fmt == kF16) return *(const u4*)((const uint16_t*)base + e);
  const u2 v = *(const u2*)((const uint8_t*)base + e);
  return to_f16x8(fmt, u4{v[0], v[1], 0u, 0u});
}

// Rows of a matrix of 8 bits on their way into an LDS tile of ROWS x DP: fetched into
// the registers of a workgroup, or a wave (THREADS 64), eight columns a chunk, and
// decoded and stored by arrive(). The buffer's range check makes rows past the end,
// and the columns past D, read as zeros.
template <int ROWS, int DP, int THREADS>
struct StagedTile {
  static constexpr int CH = DP / 8, N = ROWS * CH / THREADS;
  u2 r[N];
  int voff0, step;  // chunk i of a thread: voff0 + i step
  const uint8_t *base, *at;
  uint32_t pitch;
  int bytes_d, fmt;

  // first: element of row 0 (of the sequence) and column 0 (of the head)
  __device__ __forceinline__ void init(const void* data, int64_t first, int64_t ld, int D, int format) {
    fmt = format;
    at = base = (const uint8_t*)data + first;
    pitch = (uint32_t)ld;
    bytes_d = D;
    const int me = (int)threadIdx.x % THREADS, row = me / CH, ch = me % CH;
    step = THREADS / CH * (int)pitch;
    // (past the end of any buffer: a tile's rows span less than 2^31 bytes)
    voff0 = ch * 8 < D ? row * (int)pitch + ch * 8 : (int)0x80000000;
  }
  // The next tile starts at row0 (of a matrix `skip` elements on).
  __device__ __forceinline__ void seek(int64_t row0, int64_t skip = 0) { at = base + row0 * pitch + skip; }
  __device__ __forceinline__ void skip(int64_t rows) { at += rows * pitch; }
  // Loads the next tile, of which `left` rows are there, and moves on by a tile.
  __device__ __forceinline__ void begin(int left, uint8_t*, int) {
    const uint32_t bytes = left > 0 ? (uint32_t)(min(left, ROWS) - 1) * pitch + (uint32_t)bytes_d : 0u;
    const auto rs = __builtin_amdgcn_make_buffer_rsrc((void*)at, 0, (int)bytes, 0x00027000);
    at += (uint64_t)pitch * ROWS;
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = __builtin_amdgcn_raw_buffer_load_b64(rs, voff0 + i * step, 0, 0);
  }
  __device__ __forceinline__ void issue(int) const {}
  __device__ __forceinline__ void arrive(uint8_t* lds) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = (int)threadIdx.x % THREADS + i * THREADS;
      const u4 codes = {r[i][0], r[i][1], 0u, 0u};
      *(u4*)(lds + tile_off<DP>(c / CH, c % CH)) = fmt == kE4M3 ? to_f16x8(kE4M3, codes) : to_f16x8(kE5M2, codes);
    }
  }
};

// One buffer_load_dwordx4 ... lds: lane i's 16 bytes land at M0 + 16 i. (M0 has no
// other user in these kernels; a scalar write of it and a buffer load need a wait
// state between them.)
typedef int v4i __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void load_to_lds16(v4i rsrc, uint32_t voff, const uint8_t* lds) {
  const uint32_t at = (uint32_t)(uintptr_t)(ATTN_LDS const void*)lds;
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
  asm volatile(
      "s_mov_b32 m0, %0\n\ts_nop 0\n\t"
      "buffer_load_dwordx4 %1, %2, 0 offen lds"
      :
      : "s"(at), "v"(voff), "s"(rsrc)
      : "memory", "m0");
#pragma clang diagnostic pop
}
// A value that is there at this point (the compiler would else form what a branch
// may replace only behind the branch, away from the products that it hides under).
template <typename T>
__device__ __forceinline__ void held(T& x) { asm volatile("" : "+v"(x)); }
// What a wave's lanes wrote to LDS before is there for its other lanes after (a wave's
// LDS instructions are done in order; this keeps the compiler to that order).
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
// Nothing is scheduled across.
__device__ __forceinline__ void slice_end() { __builtin_amdgcn_sched_barrier(0); }
// All loads so far are done, also for the compiler's own count of them (else it
// waits for these inside the loop that uses them, and with them for that loop's).
__device__ __forceinline__ void settle_loads() { __builtin_amdgcn_s_waitcnt(0x0F70); }

__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// F16 rows of a matrix loaded straight into an LDS tile of ROWS x DP: no
// registers, and the chunks' permutation is applied to the address they are read
// from. A wave's load fills 1 KiB, the workgroup's four 4 KiB.
template <int ROWS, int DP>
struct DirectTile {
  static constexpr int CH = DP / 8, N = ROWS * CH / 256;
  uint32_t voff0, step, pitch;
  const uint8_t *base, *at;
  int bytes_d;
  v4i rs;       // of the tile under way
  uint8_t* to;

  __device__ __forceinline__ void init(const void* data, int64_t first, int64_t ld, int D, int) {
    base = (const uint8_t*)data + first * 2;
    pitch = (uint32_t)(ld * 2);
    bytes_d = D * 2;
    const int row = (int)threadIdx.x / CH, slot = (int)threadIdx.x % CH;
    const int ch = (tile_off<DP>(row, slot) - row * DP * 2) >> 4;
    step = 256 / CH * pitch;
    voff0 = ch * 8 < D ? row * pitch + ch * 16 : 0x80000000u;
  }
  __device__ __forceinline__ void seek(int64_t row0, int64_t skip = 0) { at = base + row0 * pitch + 2 * skip; }
  // The next tile, of which `left` rows are there: begin(), then issue(0) ... issue(N -
  // 1). (A burst of them stops the wave until the memory pipe has taken it; one in
  // each slice of a block of products is hidden.)
  __device__ __forceinline__ void begin(int left, uint8_t* lds, int wave) {
    const uint32_t bytes = left > 0 ? (uint32_t)(min(left, ROWS) - 1) * pitch + (uint32_t)bytes_d : 0u;
    rs = v4i{(int)(uint32_t)(uintptr_t)at, (int)(uint32_t)((uint64_t)(uintptr_t)at >> 32), (int)bytes, 0x00027000};
    to = lds + wave * 1024;
    at += (uint64_t)pitch * ROWS;
  }
  __device__ __forceinline__ void issue(int i) const { load_to_lds16(rs, voff0 + i * step, to + i * 4096); }
  __device__ __forceinline__ void arrive(uint8_t*) const { wait_loads(); }
};
// The same for a wave's own tile of 32 rows: a load covers so few rows that the
// chunks' permutation differs from one to the next, with a period of four.
template <int DP>
struct WaveTile {
  static constexpr int CH = DP / 8, PER = 64 / CH, N = 32 / PER;
  uint32_t voff[4], pitch;
  const uint8_t* at;
  int bytes_d;

  __device__ __forceinline__ void init(const void* data, int64_t first, int64_t ld, int D, int) {
    at = (const uint8_t*)data + first * 2;
    pitch = (uint32_t)(ld * 2);
    bytes_d = D * 2;
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int row = k * PER + lane / CH, ch = (tile_off<DP>(row, lane % CH) - row * DP * 2) >> 4;
      voff[k] = ch * 8 < D ? row * pitch + ch * 16 : 0x80000000u;
    }
  }
  __device__ __forceinline__ void skip(int64_t rows) { at += rows * pitch; }
  __device__ __forceinline__ void begin(int left, uint8_t* lds, int) {
    const uint32_t bytes = left > 0 ? (uint32_t)(min(left, 32) - 1) * pitch + (uint32_t)bytes_d : 0u;
    const v4i rs = {(int)(uint32_t)(uintptr_t)at, (int)(uint32_t)((uint64_t)(uintptr_t)at >> 32), (int)bytes, 0x00027000};
#pragma unroll
    for (int i = 0; i < N; ++i) load_to_lds16(rs, voff[i & 3] + (i >> 2) * 4 * PER * pitch, lds + i * 1024);
    at += (uint64_t)pitch * 32;
  }
  __device__ __forceinline__ void arrive(uint8_t*) const { wait_loads(); }
};
// A tile whose matrix is F16, or has 8 bits.
template <bool F16, int ROWS, int DP>
using Tile = typename std::conditional<F16, DirectTile<ROWS, DP>, StagedTile<ROWS, DP, 256>>::type;

// Operand with one row of the tile a lane (rows row0 + (lane & 31)), k = columns
// 16 ks + 8 h ...
template <int DP>
__device__ __forceinline__ h8 row_operand(const uint8_t* lds, int row0, int ks, int lane) {
  return *(const h8*)(lds + row0 * (DP * 2) + (tile_off<DP>(lane & 31, lane >> 5) ^ (ks << 5)));
}

// Operand with one column of the tile a lane (columns 32 db + (lane & 31)), k = rows
// row0 .. row0 + 15 in the order of a result's registers. row0: a multiple of 16.
template <int DP>
__device__ __forceinline__ h8 col_operand(const uint8_t* lds, int row0, int db, int lane) {
  const int h = lane >> 5, x = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
  const int row = 4 * h + ((lane & 15) >> 2);
  const int a0 = (tile_off<DP>(row, x) ^ (db << 6)) + 8 * (lane & 1);
  const int a1 = (tile_off<DP>(row + 8, x) ^ (db << 6)) + 8 * (lane & 1);
  const uint8_t* t = lds + row0 * (DP * 2);
  const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ATTN_LDS s4*)(t + a0));
  const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ATTN_LDS s4*)(t + a1));
  typedef short s8 __attribute__((ext_vector_type(8)));
  return __builtin_bit_cast(h8, (s8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// The same from global memory, for the whole kernel: the row that starts at element
// e (columns from D on, and rows that are not there, zero).
template <int KS>
__device__ __forceinline__ void load_row_operands(int fmt, const void* base, int64_t e, int h, int D, bool ok, h8 (&v)[KS]) {
  u4 w[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) w[ks] = u4{0u, 0u, 0u, 0u};
  if (fmt == kF16) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      if (ok && 16 * ks + 8 * h < D) w[ks] = *(const u4*)((const uint16_t*)base + e + 16 * ks + 8 * h);
  } else {
    u2 b[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      b[ks] = u2{0u, 0u};
      if (ok && 16 * ks + 8 * h < D) b[ks] = *(const u2*)((const uint8_t*)base + e + 16 * ks + 8 * h);
    }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) w[ks] = to_f16x8(fmt, u4{b[ks][0], b[ks][1], 0u, 0u});
  }
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) v[ks] = __builtin_bit_cast(h8, w[ks]);
}

__device__ __forceinline__ f16v mfma(h8 a, h8 b, f16v c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// Registers 8 g ... 8 g + 7 of a result as an operand (round to nearest even).
template <typename Values>
__device__ __forceinline__ h8 to_operand(const Values& x, int g) {
  h8 r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = (_Float16)x[8 * g + i];
  return r;
}

// Row of a result held in register r of a lane of half h.
__device__ __forceinline__ int result_row(int r, int h) { return 8 * (r >> 2) + 4 * h + (r & 3); }

// The other half's value (lane ^ 32).
__device__ __forceinline__ float other_half(float x, int h) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(h ? r[0] : r[1]);
}

// Whether an operand holds an infinity or NaN.
__device__ __forceinline__ bool not_finite(h8 v) {
  const u4 w = __builtin_bit_cast(u4, v);
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m = max(m, w[i] & 0x7C000000u);
    m = max(m, (w[i] << 16) & 0x7C000000u);
  }
  return m == 0x7C000000u;
}

// v with infinities and NaN replaced by 0.
__device__ __forceinline__ h8 finite_part(h8 v) {
  u4 w = __builtin_bit_cast(u4, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if ((w[i] & 0x7C000000u) == 0x7C000000u) w[i] &= 0xFFFFu;
    if ((w[i] & 0x7C00u) == 0x7C00u) w[i] &= 0xFFFF0000u;
  }
  return __builtin_bit_cast(h8, w);
}

// A wave's result of 32 rows (a row a lane pair, columns over the registers) times f,
// 0 where f is, through `lds` (32 rows of DP floats, the wave's own) so that whole rows
// are stored: to fp32 where f32 is given, else to codes. place(row, e32, e): the element
// of a row's first column in either. Returns the largest magnitude of the lane's row.
// (Stored from the registers, 16 bytes of 32 rows at a time, dK and dV of 128 keys
// took 26000 clocks, as much as the products of six tiles.)
template <int DP, typename PlaceOf>
__device__ __forceinline__ float store_rows(uint8_t* lds, const f16v (&acc)[DP / 32], float f, int lane, int rows, int D, float* f32,
                                            void* codes, int fmt, int shift, bool sat, PlaceOf place) {
  constexpr int CH = DP / 16, MASK = DP / 4 - 1;
  const int h = lane >> 5, r = lane & 31;
  float a = 0.0f;
  wave_sync();
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        y[i] = f == 0.0f ? 0.0f : acc[d][4 * g + i] * f;
        a = fmaxf(a, fabsf(y[i]));  // (fmaxf skips NaN)
      }
      *(float4*)(lds + r * DP * 4 + (((8 * d + 2 * g + h) ^ (r & MASK)) << 4)) = make_float4(y[0], y[1], y[2], y[3]);
    }
  wave_sync();
  const bool fast = shift >= kFastShiftMinSub && shift <= kFastShiftMax;
  const float scale = fast ? pow2_float(shift) : 1.0f;
  const int c = lane % CH;
#pragma unroll 1
  for (int row = lane / CH; row < 32; row += 64 / CH) {
    if (row >= rows || 16 * c >= D) continue;
    int64_t e32, e;
    place(row, e32, e);
    uint32_t u[16], w[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const u4 x = *(const u4*)(lds + row * DP * 4 + (((4 * c + k) ^ (row & MASK)) << 4));
      u[4 * k] = x[0];
      u[4 * k + 1] = x[1];
      u[4 * k + 2] = x[2];
      u[4 * k + 3] = x[3];
      if (f32) *(u4*)(f32 + e32 + 16 * c + 4 * k) = x;
    }
    if (f32) continue;
    if (fmt == kF16) {
      encode16<kF16>(u, shift, scale, fast, sat, w);
      store_words16<kF16>(codes, e + 16 * c, w);
    } else if (fmt == kE4M3) {
      encode16<kE4M3>(u, shift, scale, fast, sat, w);
      store_words16<kE4M3>(codes, e + 16 * c, w);
    } else {
      encode16<kE5M2>(u, shift, scale, fast, sat, w);
      store_words16<kE5M2>(codes, e + 16 * c, w);
    }
  }
  return r < rows ? a : 0.0f;
}

// A pair that the mask does not admit has weight 0, and 0 * Inf must add
// nothing. Only tiles that a mask cuts hold such pairs next to admitted ones. A
// tile of those that holds an infinity or NaN is marked (`flag`: the tile's number, so
// it needs no clearing; 256 threads, whose barrier the caller owes); its finite part is
// then multiplied as usual, and the rest added pair by pair.
template <int ROWS, int DP>
__device__ __forceinline__ void mark_not_finite(const uint8_t* tile, int* flag, int number) {
  bool bad = false;
  for (int i = threadIdx.x; i < ROWS * DP / 8; i += 256) bad |= not_finite(((const h8*)tile)[i]);
  if (bad) *flag = number;
}

__device__ __forceinline__ float f16_bits(uint32_t b) { return (float)__builtin_bit_cast(_Float16, (uint16_t)b); }

// v where it is an infinity or NaN, else 0.
__device__ __forceinline__ float odd_part(uint32_t b) { return (b & 0x7C00u) == 0x7C00u ? f16_bits(b) : 0.0f; }

// Four consecutive values of a row, cast to a format with a shift, at element e.
__device__ __forceinline__ void store4_any(int fmt, void* base, int64_t e, const float (&y)[4], int shift, bool sat) {
  const bool fast = shift >= kFastShiftMinSub && shift <= kFastShiftMax;
  uint32_t u[4];
  bool nan = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    u[i] = __float_as_uint(y[i]);
    nan |= is_nan_bits(u[i]);
  }
  const bool hw = fast && !nan;
  if (fmt == kF16) {
    u2 w;
    const float inv = fast ? pow2_float(-shift) : 1.0f;
    w[0] = hw ? cast2_f16_hw(u[0], u[1], inv, sat) : cast2_exact_f16(u[0], u[1], shift, sat);
    w[1] = hw ? cast2_f16_hw(u[2], u[3], inv, sat) : cast2_exact_f16(u[2], u[3], shift, sat);
    *(u2*)((uint16_t*)base + e) = w;
  } else if (fmt == kE4M3) {
    *(uint32_t*)((uint8_t*)base + e) = hw ? cast4_fp8_hw<kE4M3>(u[0], u[1], u[2], u[3], pow2_float(shift), sat)
                                          : cast4_exact_fp8<kE4M3>(u[0], u[1], u[2], u[3], shift, sat);
  } else {
    *(uint32_t*)((uint8_t*)base + e) = hw ? cast4_fp8_hw<kE5M2>(u[0], u[1], u[2], u[3], pow2_float(shift), sat)
                                          : cast4_exact_fp8<kE5M2>(u[0], u[1], u[2], u[3], shift, sat);
  }
}

// Factor of the scores in powers of two: alpha s_q s_k log2 e, held to where its
// inverse and its product with any score are finite (a score of F16 data lies under
// 2^39 and, where it is not 0, over 2^-48).
__device__ __forceinline__ float score_factor(const AttnParams& p) {
  const float f = __builtin_ldexpf(p.alpha, pow2_exponent(p.s_q) + pow2_exponent(p.s_k)) * kLog2e;
  return fminf(fmaxf(f, 0x1p-100f), 0x1p80f);
}

// Position in the grid of `per_head` workgroups for each (sequence, key head). A
// head's workgroups read the same rows (keys, or the queries of the backward) while
// they run side by side, so they go to one XCD, whose L2 then serves them:
// workgroups are dealt to the eight XCDs in turn, and where the heads are a
// multiple of 8, XCD x takes heads x, x + 8, ..., four at a time and of these the
// longest workgroups first. (4 x 4096 causal tokens, 32 heads of 128: forward 672 us
// with one head at a time, whose last workgroups find CUs busy with long ones, 664
// with two, 641 with four, 644 with eight, 662 with all 16; dK and dV 1517, 1481, 1474
// and 1486 us with one, two, four and eight.) Else the head runs fastest.
constexpr int kHeadsAtOnce = 4;
struct Place {
  int64_t b;
  int hk;
  int64_t rest;
};
__device__ __forceinline__ Place attn_place(const AttnParams& p, int64_t in_head) {
  // (32 bits: a call has less than 2^31 workgroups)
  const uint32_t heads = (uint32_t)(p.batch * p.Hkv), per_head = (uint32_t)in_head, id = p.group0 + blockIdx.x;
  uint32_t bh;
  Place w;
  if ((heads & 7) == 0) {
    const uint32_t s = id >> 3, group = s / (per_head * kHeadsAtOnce);
    const uint32_t r = s - group * per_head * kHeadsAtOnce, n = min((uint32_t)kHeadsAtOnce, heads / 8 - group * kHeadsAtOnce);
    w.rest = r / n;
    bh = 8 * (group * kHeadsAtOnce + r - (uint32_t)w.rest * n) + (id & 7);
  } else {
    w.rest = id / heads;
    bh = id - (uint32_t)w.rest * heads;
  }
  w.b = bh / (uint32_t)p.Hkv;
  w.hk = (int)(bh - (uint32_t)w.b * p.Hkv);
  return w;
}

}  // namespace scalify
