// F16 matrix product of the losses for gfx950, its epilogues fused: the logits
// z = x w^T with their row statistics (forward) or their gradient (backward), and
// the products dx = dz w and dw = dz^T x. 8-bit operands are F16 values and come
// decoded; all sums are fp32.
//
// Bound: the matrix instructions (2 M N K operations; a workgroup reads 64 KiB for
// 8.4e6 of them). The arrangement is that of gemm4_kernel.h, whose tiles have the
// same bytes (64 k of F16 instead of 128 of FP8): one workgroup of four waves a CU
// walks its tiles of 256 x 256, a wave holds 128 x 128 of them in AGPRs, loads go
// straight to LDS two steps ahead, over the end of a tile into the next one.
// Operands whose k is contiguous ("KC", 128-byte rows) are read with ds_read_b128,
// the others ("MC", 64 k-rows of 512 bytes) with the transposing ds_read_b64_tr_b16.
//
// Measured, 16384 x 32000 x 4096 with 8-bit w: logits and statistics 2830-2880 us (1490-1520
// TFLOP/s; library products of F16 reach 1366-1415 with both operands along k), dz 3160 (1357),
// dx 3100 (1384; library 1199-1344), dw in fp32 2950 (1457; library 1062-1071). The epilogues
// stop the matrix cores (about 7 % of the three products), which else run at the power limit.
// 256 x 256 tiles need 256 of them to fill the device: 125 (150 rows against 32000) leave
// half of it idle, 55 us for 2048 columns.
#pragma once
#include "gemm4_kernel.h"
#include "loss_dev.h"

namespace scalify {

constexpr int LK = 64;  // k of a step
typedef _Float16 lh2 __attribute__((ext_vector_type(2)));
typedef short ls4 __attribute__((ext_vector_type(4)));

// MC tiles: 16-byte chunks of a k-row are permuted in pairs, so that the four rows
// of a transposing read of 16 lanes, and those of its neighbour, meet distinct banks.
__device__ __forceinline__ int swz_mc16(int k) { return 2 * ((k & 3) | (((k >> 4) & 1) << 2)); }

// The same for 8 bits (rows of 256 bytes): eight rows of a transposing read, and their neighbour's.
__device__ __forceinline__ int swz_mc8(int k) { return (k & 7) | (((k >> 4) & 1) << 3); }

// A wave's operands in LDS. Part S (32 k of a step) of the operand of 16 rows or
// columns 16 i .. of the wave's tile: lane l serves row or column l & 15, k = 16
// (l >> 4) + 8 S .. + 7 (any order does that both operands share). A lane's address
// of part 0, i = 0 (wave_first: the wave's first row or column in the tile):
template <bool MC>
__device__ __forceinline__ uint32_t operand_addr(int wave_first, int lane) {
  const int t = lane & 15, g = lane >> 4;
  if constexpr (MC) {
    const int k = 16 * g + (t >> 2);
    return (uint32_t)(k * 512 + 2 * wave_first + swz_mc16(k) * 16 + ((t & 3) >> 1) * 16 + (t & 1) * 8);
  } else {
    return (uint32_t)((wave_first + t) * 128 + (((2 * g) ^ swz_kc(t)) * 16));
  }
}
// Read Q of an operand (both parts; KC 2 reads, MC 4). The permutations are of the
// lane alone, so i and the part only move the address, or flip bits of it.
template <bool MC, int I, int Q>
__device__ __forceinline__ void read_part(v4i (&f)[2], const uint8_t* lds, uint32_t addr) {
  if constexpr (MC) {
    constexpr int S = Q / 2, H = Q % 2;
    const ls4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS ls4*)(lds + (addr ^ (32 * I)) + 4096 * S + 2048 * H));
    const v2i w = __builtin_bit_cast(v2i, v);
    f[S][2 * H] = w.x;
    f[S][2 * H + 1] = w.y;
  } else {
    f[Q] = *(const v4i*)(lds + (addr ^ (16 * Q)) + 2048 * I);
  }
}

// Sum or maximum over the four lanes that hold a row (lane ^ 16, lane ^ 32).
template <typename F>
__device__ __forceinline__ float row4(float v, F f) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float row4_max(float v) {
  return row4(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float row4_sum(float v) {
  return row4(v, [](float a, float b) { return a + b; });
}

// A value that the compiler forms anew from here on (the flipped addresses would
// else each stay in a register over the whole loop).
__device__ __forceinline__ void held(uint32_t& x) { asm volatile("" : "+v"(x)); }

// OF: what LOSS_DW stores, a format's codes or a LossForm.
// BF: b's rows are F16 (kF16), or codes of 8 bits (whole groups of 16 of them): they lie in
// LDS as they are (KC 256 rows of 64 bytes, MC 64 k-rows of 256, read with
// ds_read_b64_tr_b8) and are decoded between products, two a product, while the group
// before theirs is multiplied.
template <bool A_MC, bool B_MC, int EPI, int OF, int BF = kF16>
__global__ __launch_bounds__(256, 1) void loss_gemm_kernel(LossGemm p) {
  using C = WaveCfg<4>;
  constexpr int WTM = C::WTM, WTN = C::WTN, MI = C::MI, NI = C::NI, BPW = C::BPW;
  constexpr bool B8 = BF != kF16;
  constexpr int BPB = B8 ? BPW / 2 : BPW;  // a wave's loads of b a step
  // bytes of an element that goes through LDS, and of a wave's 16 rows
  constexpr int ESZ = EPI == LOSS_DZ ? 2 : (EPI != LOSS_DW ? 4 : (OF == FORM_F32 ? 4 : (OF == kF16 || OF == FORM_STICKY ? 2 : 1)));
  constexpr int STAGE = EPI == LOSS_STATS || EPI == LOSS_DX ? 0 : 2048 * ESZ;
  // stores of an epilogue whose tile lies inside the matrix, at least
  constexpr int STORES = EPI == LOSS_DZ ? 32 : (EPI == LOSS_DW ? 16 * ESZ : 0);
  // [A of even steps | A of odd steps | B | B | the waves' staging]
  __shared__ __attribute__((aligned(1024))) uint8_t smem[4 * TILE_BYTES + 4 * STAGE];

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = gridDim.x;
  const int count = (int)p.hdr[LOSS_COUNT];
  const int M = p.count_is == 0 ? count : p.M, N = p.N, K = p.count_is == 1 ? count : p.K;
  const int tiles_m = (M + BM - 1) / BM, tiles_n = (N + BN - 1) / BN;
  const int T1 = tiles_m * tiles_n, T = T1 * p.splits;
  const int ntiles = (T - (int)blockIdx.x + G - 1) / G;
  if (ntiles <= 0) return;
  const int k_span = p.splits > 1 ? ((K + p.splits - 1) / p.splits + 127) / 128 * 128 : K;
  const int KT = (k_span + LK - 1) / LK;
  const int KTe = KT < 2 ? 2 : KT + (KT & 1);  // steps a tile, even
  const uint32_t lda = (uint32_t)p.lda, ldb = (uint32_t)p.ldb;

  uint32_t qa[BPW], qb[BPW];
  int kc[2], kc8 = 0;
#pragma unroll
  for (int q = 0; q < BPW; ++q) {
    const uint32_t blk = (uint32_t)(wave * BPW + q);
    // KC: 8 rows of 128 bytes a block; MC: two k-rows of 512 bytes
    const int c = (lane & 7) ^ (lane >> 3) ^ (q & 1);
    const int kr = (int)(2 * blk) + (lane >> 5);
    const uint32_t cm = (uint32_t)((lane & 31) ^ swz_mc16(kr));
    qa[q] = A_MC ? (uint32_t)kr * lda + 16u * cm : (blk * 8u + (uint32_t)(lane >> 3)) * lda + 16u * (uint32_t)c;
    qb[q] = B_MC ? (uint32_t)kr * ldb + 16u * cm : (blk * 8u + (uint32_t)(lane >> 3)) * ldb + 16u * (uint32_t)c;
    if (q < 2) kc[q] = 8 * c;
    if (B8 && B_MC && q < BPB) {  // 4 k-rows of 256 bytes a block
      const int row = 4 * (wave * BPB + q) + (lane >> 4);
      qb[q] = (uint32_t)row * ldb + 16u * (uint32_t)((lane & 15) ^ swz_mc8(row));
    } else if (B8 && q < BPB) {  // 16 rows of 64 bytes a block
      const int c8 = (lane & 3) ^ ((lane >> 4) & 3);
      qb[q] = (uint32_t)((wave * BPB + q) * 16 + (lane >> 2)) * ldb + 16u * (uint32_t)c8;
      kc8 = 16 * c8;
    }
  }

  // The call's operands, read anew by the scalar unit where a tile needs them: held over the
  // loop they would not fit the scalar registers.
  typedef const __attribute__((address_space(4))) LossGemm* Args;
  auto fresh_args = [&]() {
    Args a = (Args)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(a));
    return a;
  };
  // Tile r of this workgroup: split and origin.
  auto origin = [&](int r, int& m0, int& n0, int& split) {
    const int t = (int)blockIdx.x + r * G;
    split = p.splits > 1 ? t / T1 : 0;
    tile_origin(t - split * T1, tiles_m, tiles_n, m0, n0);
  };
  // Load cursor: the (tile, step) whose loads go out next; k l_k up to l_end. A KC
  // operand's buffer starts at the tile's first row, an MC operand's at the step's
  // first k-row; both end with the matrix, and loads past that, or past l_end, read
  // zeros.
  int l_r = 0, l_kt = 0, l_k, l_end;
  v4i ra, rb;
  const uint8_t *la, *lb;  // MC: the step's first row
  uint32_t wa, wb;         // MC: bytes of a row that are left (rows hold whole groups of 8)
  auto rows_buffer = [&](const void* base, int64_t ld, int row0, int rows, bool codes) {
    const int n = min(rows - row0, 256);
    const uint32_t width = codes ? (uint32_t)K : 2u * (uint32_t)((K + 7) & ~7);
    return make_rsrc((const uint8_t*)base + (int64_t)row0 * ld, (uint32_t)((int64_t)(n - 1) * ld) + width);
  };
  auto k_buffer = [&](const uint8_t* base, uint32_t ld, uint32_t width) {
    const int n = min(l_end - l_k, LK);
    return make_rsrc(base, n > 0 ? (uint32_t)(n - 1) * ld + width : 0u);
  };
  auto load_tile = [&]() {
    const auto& p = *fresh_args();
    int m0, n0, split;
    origin(l_r, m0, n0, split);
    l_k = split * k_span;
    l_end = min(K, l_k + k_span);
    if constexpr (A_MC) {
      la = (const uint8_t*)p.a + (int64_t)l_k * p.lda + 2 * (int64_t)m0;
      wa = 2u * (uint32_t)(((M + 7) & ~7) - m0);
      ra = k_buffer(la, lda, wa);
    } else {
      ra = rows_buffer(p.a, p.lda, m0, M, false);
    }
    if constexpr (B_MC) {
      lb = (const uint8_t*)p.b + (int64_t)l_k * p.ldb + (B8 ? 1 : 2) * (int64_t)n0;
      wb = B8 ? (uint32_t)(((N + 15) & ~15) - n0) : 2u * (uint32_t)(((N + 7) & ~7) - n0);
      rb = k_buffer(lb, ldb, wb);
    } else {
      rb = rows_buffer(p.b, p.ldb, n0, N, B8);
    }
  };
  load_tile();
  auto advance = [&]() {
    l_k += LK;
    if (++l_kt == KTe) {
      l_kt = 0;
      if (++l_r < ntiles) {
        load_tile();
        return;
      }
      l_k = l_end;  // (and on from there: nothing is left)
    }
    if constexpr (A_MC) {
      la += (uint64_t)lda * LK;
      ra = k_buffer(la, lda, wa);
    }
    if constexpr (B_MC) {
      lb += (uint64_t)ldb * LK;
      rb = k_buffer(lb, ldb, wb);
    }
  };
  // Load j of a step into its stage P: j < BPW are A blocks, the rest B blocks.
  auto issue_one = [&](int j, int P) {
    const bool is_a = j < BPW;
    const int q = is_a ? j : j - BPW;
    uint32_t off = is_a ? qa[q] : qb[q];
    if (!is_a && B8 && !B_MC) {
      off += (uint32_t)l_k;
      if (l_k + kc8 >= l_end) off = 0x80000000u;
    } else if (!(is_a ? A_MC : B_MC)) {
      off += 2u * (uint32_t)l_k;
      if (l_k + kc[q & 1] >= l_end) off = 0x80000000u;
    }
    load_lds16(is_a ? ra : rb, off, smem + (is_a ? P : 2 + P) * TILE_BYTES + (wave * (is_a ? BPW : BPB) + q) * 1024);
  };

  const int wm = (wave / C::WAVES_N) * WTM;
  const int wn = (wave % C::WAVES_N) * WTN;
  constexpr int DSA = A_MC ? 4 : 2, DSB = (B_MC ? 4 : 2) / (B8 ? 2 : 1);
  constexpr int H = 6;
  constexpr int TS = (NI - H) * MI, AS = (H - 1) * MI, BP = 2 * DSB;
  constexpr int RX = MI < (NI - 2) * DSB ? MI : (NI - 2) * DSB;
  static_assert((NI - 2) * DSB <= H * MI, "head too short for its reads");
  v4i af[2][MI][2];
  v4i bf[NI][2];
  v4i raw[B8 ? NI : 1];  // a group's 16 codes of a lane
  uint32_t aa = operand_addr<A_MC>(wm, lane);
  const int t8 = lane & 15, k8 = 16 * (lane >> 4) + (t8 >> 1);
  uint32_t ab = !B8    ? operand_addr<B_MC>(wn, lane)
                : B_MC ? (uint32_t)(k8 * 256 + (((wn >> 4) ^ swz_mc8(k8)) << 4) + 8 * (t8 & 1))
                       : (uint32_t)((wn + t8) * 64 + (((lane >> 4) ^ ((lane >> 2) & 3)) << 4));
  auto read_b = [&](auto group_tag, auto part_tag, const uint8_t* lds) {
    constexpr int g = decltype(group_tag)::value;
    if constexpr (B8 && B_MC) {
      constexpr int S = decltype(part_tag)::value;
      const v2i v = __builtin_amdgcn_ds_read_tr8_b64_v2i32((LDS_AS v2i*)(lds + (ab ^ (16 * g)) + 2048 * S));
      raw[g][2 * S] = v.x;
      raw[g][2 * S + 1] = v.y;
    } else if constexpr (B8)
      raw[g] = *(const v4i*)(lds + ab + 1024 * g);
    else
      read_part<B_MC, g, decltype(part_tag)::value>(bf[g], lds, ab);
  };
  // Decodes pairs FIRST .. LAST - 1 of the codes of all groups, eight pairs a group.
  auto decode = [&](auto first_tag, auto last_tag) {
    static_for<decltype(first_tag)::value, decltype(last_tag)::value>([&](auto Q) {
      constexpr int g = decltype(Q)::value / 8, c = decltype(Q)::value % 8;
      const lh2 v = BF == kE4M3 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((uint32_t)raw[g][c >> 1], 1.0f, c & 1)
                                : __builtin_amdgcn_cvt_scalef32_pk_f16_bf8((uint32_t)raw[g][c >> 1], 1.0f, c & 1);
      int w = __builtin_bit_cast(int, v);
      // (here and no later: a product may not follow what writes its operand at once, and the
      // compiler does not see that the products are products)
      asm volatile("" : "+v"(w));
      bf[g][c >> 2][c & 3] = w;
    });
  };

  bool stored = false;  // the last thing done is an epilogue with all its stores
  // Schedule of a step: that of gemm4_kernel, with a pair of products in the place of
  // each of its products (the two k parts of 32).
  auto head = [&](auto par_tag) {
    constexpr int P = decltype(par_tag)::value;
    const uint8_t* cB = smem + (2 + P) * TILE_BYTES;
    held(ab);
    static_for<0, H * MI>([&](auto I) {
      constexpr int i = decltype(I)::value;
      constexpr int ni = i / MI, u = 2 * (i % MI), ks = u / MI, mi = u % MI;
      AccTile<mi * NI + ni>::mfma_f16(bf[ni][ks], af[P][mi][ks]);
      AccTile<(mi + 1) * NI + ni>::mfma_f16(bf[ni][ks], af[P][mi + 1][ks]);
      if constexpr (i < (NI - 2) * DSB) {
        constexpr int g = 2 + i / DSB;
        read_b(std::integral_constant<int, g>{}, std::integral_constant<int, i % DSB>{}, cB);
      }
      // (groups 1 .. NI - 1, each done before its first product)
      if constexpr (B8) decode(std::integral_constant<int, 8 + i * 8 * (NI - 1) / (H * MI)>{}, std::integral_constant<int, 8 + (i + 1) * 8 * (NI - 1) / (H * MI)>{});
      if constexpr (i == MI - 1) {
        wait_lgkmcnt<RX>();
        __builtin_amdgcn_s_barrier();
      }
      if constexpr (i >= MI) {
        constexpr int j = i - MI;
        static_for<j * BPW / AS, (j + 1) * BPW / AS>([&](auto J) { issue_one(decltype(J)::value, P); });
      }
    });
    // (vector memory is done in order: behind an epilogue's stores, the loads of the next
    // step are older than they are)
    if (STORES > 0 && P == 0 && stored)
      wait_vmcnt<(BPW + STORES < 63 ? BPW + STORES : 63)>();
    else
      wait_vmcnt<BPW>();
    stored = false;
    wait_lgkmcnt<0>();
    __builtin_amdgcn_s_barrier();
  };
  auto tail = [&](auto par_tag) {
    constexpr int P = decltype(par_tag)::value;
    const uint8_t* nA = smem + (P ^ 1) * TILE_BYTES;
    const uint8_t* nB = smem + (2 + (P ^ 1)) * TILE_BYTES;
    held(aa);
    held(ab);
    static_assert(NI - H == 2, "a slot of the tail is a k part of a row of tiles");
    static_for<0, TS>([&](auto I) {
      constexpr int i = decltype(I)::value;
      constexpr int ks = i % 4 / 2, mi = 2 * (i / 4) + i % 2;
      AccTile<mi * NI + H>::mfma_f16(bf[H][ks], af[P][mi][ks]);
      AccTile<mi * NI + H + 1>::mfma_f16(bf[H + 1][ks], af[P][mi][ks]);
      static_for<i * BPB / TS, (i + 1) * BPB / TS>([&](auto J) { issue_one(BPW + decltype(J)::value, P); });
      if constexpr (B8) {
        if constexpr (i < BP) read_b(std::integral_constant<int, i / DSB>{}, std::integral_constant<int, i % DSB>{}, nB);
        constexpr int first = i - (TS - 10);  // (done two slots before the head's first product)
        if constexpr (first >= 0 && first < 8) decode(std::integral_constant<int, first>{}, std::integral_constant<int, first + 1>{});
      } else {
        static_for<i * BP / TS, (i + 1) * BP / TS>([&](auto Q) {
          constexpr int q = decltype(Q)::value;
          read_b(std::integral_constant<int, q / DSB>{}, std::integral_constant<int, q % DSB>{}, nB);
        });
      }
      static_for<i * (MI * DSA) / TS, (i + 1) * (MI * DSA) / TS>([&](auto Q) {
        constexpr int q = decltype(Q)::value;
        read_part<A_MC, q / DSA, q % DSA>(af[P ^ 1][q / DSA], nA, aa);
      });
    });
    advance();
  };

  // ---- epilogues: a lane holds C[m][n .. n + 3] of tile (mi, ni) at m = m0 + wm +
  // 16 mi + (lane & 15), n = n0 + wn + 16 ni + 4 (lane >> 4)
  uint8_t* const st = smem + 4 * TILE_BYTES + wave * STAGE;
  const int lr = lane & 15, lq = lane >> 4;
  float lmax = 0.f;
  int d_shift = 0, e_out = 0;
  bool d_fast = false;
  float d_scale = 1.0f, d_inv = 1.0f;
  if constexpr (EPI == LOSS_DW) {
    if constexpr (OF != FORM_F32 && OF != FORM_STICKY) {  // the scale is known: codes at once
      const int unit = hdr_weight(p.hdr) - kLossGradLog2;
      const int base = pow2_exponent(p.s0) + pow2_exponent(p.s1);
      e_out = clamp_e8m0(base);
      d_shift = e_out - base - unit;
      d_fast = d_shift >= kFastShiftMinSub && d_shift <= kFastShiftMax;
      if (d_fast) d_scale = pow2_float(d_shift), d_inv = pow2_float(-d_shift);
    }
  }
  // A tile's numbers of a lane's rows, loaded while its last steps run.
  float r_f[MI], r_l[MI], r_c[MI];
  int r_i[MI];  // label; LOSS_PICK: row
  int r_e[MI], bin_lo = 0, bin_hi = 0;  // LOSS_PICK: a lane's entry; lane mi: the rows' first entry and the end
  auto load_bins = [&](int m0, int n0) {
    if constexpr (EPI == LOSS_PICK) {
      const auto& p = *fresh_args();
      const int group = (m0 + wm) / 16 + (lane & (MI - 1));
      const int* o = p.bins + (int64_t)group * (p.bin_columns + 1) + (n0 + wn) / WTN;
      const bool there = 16 * group < M && n0 + wn < N;
      bin_lo = there ? o[0] : 0;
      bin_hi = there ? o[1] : 0;
    }
  };
  auto load_rows = [&](int m0) {
    if constexpr (EPI != LOSS_DW) {
      const auto& p = *fresh_args();
#pragma unroll
      for (int mi = 0; mi < MI; ++mi) {
        const int m = min(m0 + wm + 16 * mi + lr, M - 1);
        r_f[mi] = EPI == LOSS_DX ? p.dx_factor[m] : p.factor[m];
        if constexpr (EPI == LOSS_DX) continue;
        if constexpr (EPI == LOSS_DZ) r_l[mi] = p.lse2[m], r_c[mi] = p.coef[m];
        if constexpr (EPI == LOSS_PICK) {
          r_i[mi] = p.rows[m];
          const int at = __builtin_amdgcn_readlane(bin_lo, mi) + lane;
          r_e[mi] = at < __builtin_amdgcn_readlane(bin_hi, mi) ? p.entries[(int64_t)((m0 + wm) / 16 + mi) * 16 * p.top + at] : 0;
        } else
          r_i[mi] = p.label ? p.label[m] : -1;
      }
    }
  };
  // The 32 values of a lane's row (mi) of the wave's tile, and the accumulators back to 0.
  auto take = [&](auto mi_tag, float (&x)[4 * NI]) {
    constexpr int mi = decltype(mi_tag)::value;
    static_for<0, NI>([&](auto J) {
      constexpr int ni = decltype(J)::value;
      const v4f v = AccTile<mi * NI + ni>::read();
      AccTile<mi * NI + ni>::zero();
#pragma unroll
      for (int i = 0; i < 4; ++i) x[4 * ni + i] = v[i];
    });
  };
  // 16 rows of a wave's 128 columns through its LDS (the 16-byte chunks of a row permuted
  // by the row), so that whole rows are stored: group(ni) gives a lane's four elements.
  constexpr int CPR = 8 * ESZ;  // chunks of a row
  auto stage_rows = [&](auto group) {
    static_for<0, NI>([&](auto Q) {
      constexpr int ni = decltype(Q)::value;
      const int chunk = ESZ == 4 ? 4 * ni + lq : (ESZ == 2 ? 2 * ni + (lq >> 1) : ni);
      const int off = ESZ == 4 ? 0 : (ESZ == 2 ? 8 * (lq & 1) : 4 * lq);
      const auto w = group(Q);
      *(std::remove_const_t<decltype(w)>*)(st + lr * 16 * CPR + ((chunk ^ (lr & (CPR - 1))) * 16) + off) = w;
    });
    wait_lgkmcnt<0>();
  };
  // They go to rows m0 .. and columns n0 .. (below cols) of a matrix of pitch ld.
  auto store_rows = [&](void* base, int64_t ld, int m0, int n0, int cols) {
    constexpr int ROWS = 64 / CPR, PER = 16 / ESZ;
    u4 o[16 / ROWS];
#pragma unroll
    for (int j = 0; j < 16 / ROWS; ++j) {
      const int r = ROWS * j + lane / CPR, c = lane % CPR;
      o[j] = *(const u4*)(st + r * 16 * CPR + ((c ^ (r & (CPR - 1))) * 16));
    }
    wait_lgkmcnt<0>();
#pragma unroll
    for (int j = 0; j < 16 / ROWS; ++j) {
      const int row = m0 + ROWS * j + lane / CPR, col = n0 + PER * (lane % CPR);
      uint8_t* to = (uint8_t*)base + ((int64_t)row * ld + col) * ESZ;
      if (row < M && col < cols) {
        if (EPI != LOSS_DW || OF == FORM_F32 || OF == FORM_STICKY || col + PER <= cols) {  // (pitches of whole chunks)
          *(u4*)to = o[j];
        } else {
#pragma unroll
          for (int i = 0; i < PER - 1; ++i)
            if (col + i < cols) {
              if constexpr (ESZ == 2)
                ((uint16_t*)to)[i] = (uint16_t)(o[j][i / 2] >> (16 * (i % 2)));
              else if constexpr (ESZ == 1)
                to[i] = (uint8_t)(o[j][i / 4] >> (8 * (i % 4)));
            }
        }
      }
    }
  };
  auto store_tile = [&](int m0, int n0, int split) {
    stored = m0 + wm + WTM <= M && n0 + wn + WTN <= N;
    const auto& p = *fresh_args();
    uint32_t first_n = (uint32_t)(n0 + wn + 4 * lq);
    const bool all_n = n0 + wn + WTN <= N;
    static_for<0, MI>([&](auto J) {
      constexpr int mi = decltype(J)::value;
      const int m = m0 + wm + 16 * mi + lr;
      const bool in = m < M;
      float x[4 * NI];
      take(J, x);
      held(first_n);  // (the masks of its columns would else be kept from row to row)
      const int nb = (int)first_n;
      if constexpr (EPI == LOSS_STATS || EPI == LOSS_PICK) {
        const float f = r_f[mi];
        if (!all_n) {
#pragma unroll
          for (int i = 0; i < 4 * NI; ++i)
            if (nb + 16 * (i >> 2) + (i & 3) >= N) x[i] = -__builtin_inff();
        }
        if constexpr (EPI == LOSS_STATS) {
          const int d = in ? r_i[mi] - (p.v0 + nb) : -1;
          // (the lane that has the label's column: d = 16 ni + i)
          const bool mine = d >= 0 && d < WTN && (d & 15) < 4;
          if (__ballot(mine)) {
            float z = 0.f;
#pragma unroll
            for (int i = 0; i < 4 * NI; ++i)
              if (d == 16 * (i >> 2) + (i & 3)) z = x[i];
            if (mine) p.picked2[m] = z * f;
          }
        } else {
          // the teacher's tokens of these rows and columns (loss_bin_kernel), if any: the rows'
          // logits through LDS, a lane an entry
          const int lo = __builtin_amdgcn_readlane(bin_lo, mi), hi = __builtin_amdgcn_readlane(bin_hi, mi);
          if (hi > lo) {
            static_for<0, NI>([&](auto Q) {
              constexpr int ni = decltype(Q)::value;
              *(v4f*)(st + lr * 512 + (((4 * ni + lq) ^ lr) * 16)) = v4f{x[4 * ni], x[4 * ni + 1], x[4 * ni + 2], x[4 * ni + 3]};
            });
            wait_lgkmcnt<0>();
            const float fn = f * 0.69314718055994530942f;
            for (int j = lo; j < hi; j += 64) {
              int e = r_e[mi];
              if (j > lo && j + lane < hi) e = p.entries[(int64_t)((m0 + wm) / 16 + mi) * 16 * p.top + j + lane];
              const int row = bin_row(e), d = bin_column(e);
              const float fe = __shfl(fn, row, 64);
              const int to = __shfl(r_i[mi], row, 64);
              if (j + lane < hi)
                p.picked[(int64_t)to * p.top + bin_entry(e)] = fe * *(const float*)(st + row * 512 + (((d >> 2) ^ row) * 16) + 4 * (d & 3));
            }
            wait_lgkmcnt<0>();
          }
        }
        float top = x[0];
#pragma unroll
        for (int i = 1; i < 4 * NI; ++i) top = fmaxf(top, x[i]);
        // (a factor is positive; values of -Inf alone have the sum 0, and a NaN is in the sum)
        top = row4_max(top);
        const float m2 = top == -__builtin_inff() || top != top ? 0.f : top * f;
        float less = m2;
        if (__builtin_expect(__ballot(is_large(m2)) != 0, 0)) {
          const bool large = is_large(m2);
          less = large ? 0.f : m2;
#pragma unroll
          for (int i = 0; i < 4 * NI; ++i) x[i] = large ? x[i] - top : x[i];
        }
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 4 * NI; ++i) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], f, -less));
        sum = row4_sum(sum);
        if (lq == 0 && in) p.stats[(int64_t)((p.v0 + n0 + wn) / WTN) * p.R + m] = float2{sum == 0.f ? -__builtin_inff() : m2, sum};
      } else if constexpr (EPI == LOSS_DZ) {
        float f = r_f[mi], l = r_l[mi];
        const float c = r_c[mi];
        if (__builtin_expect(__ballot(fabsf(l) >= kLargeSum) != 0, 0)) {
#pragma unroll
          for (int i = 0; i < 4 * NI; ++i) x[i] = held_log(__builtin_fmaf(x[i], f, -l), l);
          f = 1.f, l = 0.f;
        }
#pragma unroll
        for (int i = 0; i < 4 * NI; ++i) x[i] = c * __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], f, -l));
        const int d = r_i[mi] - (p.v0 + nb);  // (no label: below 0)
        if (__ballot(d >= 0 && d < WTN && (d & 15) < 4)) {
#pragma unroll
          for (int i = 0; i < 4 * NI; ++i)
            if (d == 16 * (i >> 2) + (i & 3)) x[i] -= c;
        }
        if (!all_n) {
#pragma unroll
          for (int i = 0; i < 4 * NI; ++i)
            if (nb + 16 * (i >> 2) + (i & 3) >= N) x[i] = 0.f;
        }
        stage_rows([&](auto Q) {
          constexpr int ni = decltype(Q)::value;
          const lh2 a = {(_Float16)x[4 * ni], (_Float16)x[4 * ni + 1]}, b = {(_Float16)x[4 * ni + 2], (_Float16)x[4 * ni + 3]};
          return v2i{__builtin_bit_cast(int, a), __builtin_bit_cast(int, b)};
        });
        // (ldz is a multiple of 64: a row holds every column of the tiles it reaches)
        store_rows(p.dz, p.ldz, m0 + wm + 16 * mi, n0 + wn, (int)p.ldz);
      } else if constexpr (EPI == LOSS_DX) {
        if (in) {
          const float f = r_f[mi];
          float* o = p.part + ((int64_t)split * p.part_rows + m) * p.ldp + nb;
          static_for<0, NI>([&](auto Q) {
            constexpr int ni = decltype(Q)::value;
            if (nb + 16 * ni < p.ldp) {
              v4f v = {x[4 * ni] * f, x[4 * ni + 1] * f, x[4 * ni + 2] * f, x[4 * ni + 3] * f};
              if (p.accumulate) v += *(const v4f*)(o + 16 * ni);
              *(v4f*)(o + 16 * ni) = v;
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (nb + 16 * ni + i < N) lmax = fmaxf(lmax, fabsf(v[i]));
            }
          });
        }
      } else {
        if (!all_n) {
#pragma unroll
          for (int i = 0; i < 4 * NI; ++i)
            if (nb + 16 * (i >> 2) + (i & 3) >= N) x[i] = 0.f;
        }
        if (in) {
#pragma unroll
          for (int i = 0; i < 4 * NI; ++i) lmax = fmaxf(lmax, fabsf(x[i]));
        }
        if constexpr (OF == FORM_F32) {
          stage_rows([&](auto Q) {
            constexpr int ni = decltype(Q)::value;
            return v4f{x[4 * ni], x[4 * ni + 1], x[4 * ni + 2], x[4 * ni + 3]};
          });
          store_rows(p.part + ((int64_t)split * p.part_rows + p.v0) * p.ldp, p.ldp, m0 + wm + 16 * mi, n0 + wn, (int)p.ldp);
        } else if constexpr (OF == FORM_STICKY) {
          stage_rows([&](auto Q) {
            constexpr int ni = decltype(Q)::value;
            uint32_t u[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t b = __float_as_uint(x[4 * ni + i]);
              u[i] = b | ((b & 0xFFFFu) + 0xFFFFu);  // (bit 16 is set if a lower one is)
            }
            return v2i{(int)__builtin_amdgcn_perm(u[1], u[0], 0x07060302u), (int)__builtin_amdgcn_perm(u[3], u[2], 0x07060302u)};
          });
          store_rows((uint16_t*)p.part + (int64_t)p.v0 * p.ldp, p.ldp, m0 + wm + 16 * mi, n0 + wn, (int)p.ldp);
        } else {
          // a shift outside the conversions' window: exact wherever the result is normal
          // (below, zero either way)
          if (!d_fast) {
#pragma unroll
            for (int i = 0; i < 4 * NI; ++i) x[i] = __builtin_amdgcn_ldexpf(x[i], -d_shift);
          }
          float any = 0.f;  // (NaN if there is one, or two infinities)
#pragma unroll
          for (int i = 0; i < 4 * NI; ++i) any += x[i];
          const bool nan = __ballot(any != any) != 0;
          auto emit = [&](auto nan_tag) {
            stage_rows([&](auto Q) {
              constexpr int ni = decltype(Q)::value;
              const float* y = x + 4 * ni;
              if constexpr (OF == kF16) {
                v2i w = p.sat ? cvt4_f16_fast<true>(y[0], y[1], y[2], y[3], d_inv) : cvt4_f16_fast<false>(y[0], y[1], y[2], y[3], d_inv);
                if constexpr (decltype(nan_tag)::value) {
                  uint32_t h[4] = {(uint32_t)w.x & 0xFFFFu, (uint32_t)w.x >> 16, (uint32_t)w.y & 0xFFFFu, (uint32_t)w.y >> 16};
#pragma unroll
                  for (int i = 0; i < 4; ++i)
                    if (y[i] != y[i]) h[i] = FmtTraits<kF16>::NANC | ((__float_as_uint(y[i]) >> 16) & 0x8000u);
                  w = v2i{(int)(h[0] | (h[1] << 16)), (int)(h[2] | (h[3] << 16))};
                }
                return w;
              } else {
                uint32_t w = cast4_fp8_hw<OF>(__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]),
                                              __float_as_uint(y[3]), d_scale, p.sat);
                if constexpr (decltype(nan_tag)::value) {
#pragma unroll
                  for (int i = 0; i < 4; ++i)
                    if (y[i] != y[i]) {
                      const uint32_t c = FmtTraits<OF>::NANC | ((__float_as_uint(y[i]) >> 24) & 0x80u);
                      w = (w & ~(0xFFu << (8 * i))) | (c << (8 * i));
                    }
                }
                return w;
              }
            });
          };
          if (__builtin_expect(nan, 0))
            emit(std::true_type{});
          else
            emit(std::false_type{});
          store_rows((uint8_t*)p.out + (int64_t)p.v0 * p.ldo * ESZ, p.ldo, m0 + wm + 16 * mi, n0 + wn, N);
        }
      }
    });
  };

  // ---- the first two steps of the first tile
#pragma unroll
  for (int j = 0; j < BPW + BPB; ++j) issue_one(j, 0);
  advance();
#pragma unroll
  for (int j = 0; j < BPW + BPB; ++j) issue_one(j, 1);
  advance();
  static_for<0, MI * NI>([&](auto I) { AccTile<decltype(I)::value>::zero(); });
  wait_vmcnt<BPW + BPB>();
  __syncthreads();
  static_for<0, MI * DSA>([&](auto Q) {
    constexpr int q = decltype(Q)::value;
    read_part<A_MC, q / DSA, q % DSA>(af[0][q / DSA], smem, aa);
  });
  static_for<0, BP>([&](auto Q) {
    constexpr int q = decltype(Q)::value;
    read_b(std::integral_constant<int, q / DSB>{}, std::integral_constant<int, q % DSB>{}, smem + 2 * TILE_BYTES);
  });
  if constexpr (B8) decode(std::integral_constant<int, 0>{}, std::integral_constant<int, 8>{});
  mfma_drain();

  using P0 = std::integral_constant<int, 0>;
  using P1 = std::integral_constant<int, 1>;
  int c_r = 0, c_m0, c_n0, c_split;
  origin(0, c_m0, c_n0, c_split);
  load_bins(c_m0, c_n0);
  head(P0{});
  for (int kt = 0;;) {
    kt += 2;
    if (kt == KTe) load_rows(c_m0);
    tail(P0{});
    head(P1{});
    tail(P1{});
    if (kt == KTe) {
      kt = 0;
      mfma_drain();
      store_tile(c_m0, c_n0, c_split);
      if (++c_r == ntiles) break;
      origin(c_r, c_m0, c_n0, c_split);
      load_bins(c_m0, c_n0);
      mfma_drain();  // the zeroing writes before the next products read them
    }
    head(P0{});
  }
  wait_vmcnt<0>();  // the out-of-range loads past the last tile
  if constexpr (EPI == LOSS_DW || EPI == LOSS_DX) {
    if (!p.amax) return;
    for (int off = 32; off > 0; off >>= 1) lmax = fmaxf(lmax, __shfl_xor(lmax, off, 64));
    if (lane == 0) raise_amax(p.amax, lmax);
  }
}

}  // namespace scalify
