// Internal interface of the losses from hidden states and the output matrix:
// softmax cross entropy and distillation from a teacher's top logits.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace scalify {

// How dw is stored, beside a format's codes: fp32, or the 16-bit form of fp32 that keeps an
// 8-bit rounding (sticky16); or not at all.
enum LossForm : int { FORM_F32 = 8, FORM_STICKY = 9, FORM_NONE = 10 };

// Words of the workspace header (kHeaderBytes):
enum LossWord : int {
  LOSS_COUNT = 0,   // rows that count
  LOSS_CMAX = 1,    // largest finite |upstream gradient| of them, fp32 bits
  LOSS_WEIGHT = 2,  // largest exponent of |g T| times row scale among them, plus kWeightBias (0: none)
  LOSS_AMAX_DX = 3, // statistics of the gradients' data, in the products' units
  LOSS_AMAX_DW = 4,
};

constexpr int kLossMaxTop = 256;  // teacher's entries of a row
// The gradient of the logits is kept in F16 as 2^14 c (p - q) with c = g T / 2^h below 2 in
// magnitude (so below 2^15): normal numbers down to |c (p - q)| = 2^-28. The 2^h is a row's own,
// its product's in dx is taken out again there, and x carries it into dw. A row whose |g T| lies
// 2^s below the largest leaves min(s, 8) of that to dz and the rest to x: dz then is normal down
// to 2^-20 |g T| at the least, and x, of magnitude 1, as long as s is at most 22. What s counts
// is |g T| times the row scale, a row's weight in dw. (One power of two for all rows cost a row
// 2^-24 below the largest, of 32768 tokens, all its probabilities; one for all row scales cost
// a row of 2^-26 of the largest its part of dw.)
constexpr int kLossGradLog2 = 14, kLossShare = 8, kWeightBias = 1024;

struct LossParams {
  // the call's operands
  const void *x, *w;
  int64_t ldx, ldw;
  int x_fmt, w_fmt;
  const float *s_x, *s_w, *row_scale;
  int R, V, D;
  const int64_t* labels;  // cross entropy, else NULL
  const int64_t* index;   // distillation: [R][top]
  const void* teacher;
  int64_t ldt;
  int t_fmt, top;
  const float* s_t;
  float temp;
  const float *dloss, *s_dloss;
  float *loss, *lse, *picked;
  void *dx, *dw;
  int64_t lddx, lddw;
  int dx_fmt, dw_fmt;
  float *dx_scale, *dw_scale, *amax_out;  // (a gradient that is asked for has a scale, if maybe no rows)
  int mode, target, sat;
  // workspace; rows that count stand in their order at 0 .. count - 1
  uint32_t* hdr;
  int *rows, *pos;     // [R] row of a place; place of a row, or -1
  int* top_on;         // [R] distillation: whether the row's teacher says anything
  int* label;          // [R] of places
  float *factor;       // [R] logits in base 2 are factor * (x . w)
  float *lse2, *coef;  // [R] log-sum-exp in base 2; upstream gradient over 2^h, times 2^14
  float* dx_factor;    // [R] 2^h over the power of two of the largest |g T|
  float* picked2;      // [R] label's logit in base 2
  int *bins, *entries;  // forward: the teacher's entries of 16 places by groups of 128 tokens of a piece
  int bin_columns;      // groups
  void *xc, *xw;       // F16 rows of x; times the powers of two that dz leaves to them
  int64_t ldxc;
  void* w16;           // F16 rows of a piece of w, where its columns are no whole groups of 16 bytes
  int64_t ldw16;
  int piece;           // rows of w at a time
  float2* stats;       // [2 tiles of V][R] maximum (base 2) and sum
  void* dz;            // F16 [R][ldz]
  int64_t ldz;
  float* part;         // [splits][R][ldp] products of dx
  float* dw32;         // [dw_splits][V][ldp] products of dw (dynamic rescale, or more than one split)
  int64_t ldp;
  int splits, dw_splits;
};

// Sizes that the host decides: pieces of w, splits of dx, and the bytes of a workspace.
struct LossPlan {
  int piece, splits, dw_splits;
  bool copy_w;
  int64_t ldxc, ldw16, ldz, ldp;
  size_t bytes;
};
// Also sets the workspace's pointers of p, where p is not NULL (base 256-byte aligned).
LossPlan loss_plan(int64_t R, int64_t V, int64_t D, int w_fmt, int top, bool back, bool amax, LossParams* p, void* base);

// Rows up to which a call goes by the bytes of w (loss_few.hip); the backward's dz is then
// one piece. This is where those kernels end, not where the tiles begin to win: 128 rows
// take 0.6 to 0.7 of the time of 129 (32000 x 2048 in F16: forward 36 and 61 us, backward 129
// and 201; 32000 x 4096 in E4M3 60 and 98, 215 and 300). The host knows the rows, not how many
// of them count, so a call of more rows takes the tiles however few count.
constexpr int kLossFewRows = 128;
inline bool loss_few_bwd(int64_t R, int64_t V) {
  return R <= kLossFewRows && V <= ((int64_t)1 << 22) && R * V <= ((int64_t)1 << 28);
}
hipError_t launch_loss_few_dz(const LossParams& p, hipStream_t s);
hipError_t launch_loss_few_grads(const LossParams& p, hipStream_t s);
int loss_few_groups(const LossParams& p);  // of tokens, each with statistics of its own
hipError_t launch_loss_few(const LossParams& p, hipStream_t s);
hipError_t launch_loss_fwd(const LossParams& p, hipStream_t s);
hipError_t launch_loss_bwd(const LossParams& p, hipStream_t s);

// One launch, by its own status alone (not by an error of an earlier call).
template <typename... Args>
hipError_t launch_one(void (*kernel)(Args...), int64_t groups, int threads, hipStream_t s, Args... args) {
  void* a[] = {(void*)&args...};
  const hipError_t e = hipLaunchKernel((const void*)kernel, dim3((unsigned)groups), dim3((unsigned)threads), a, 0, s);
  if (e != hipSuccess) (void)hipGetLastError();
  return e;
}

// An entry of the teacher among 16 rows and 128 columns.
__device__ __forceinline__ int bin_pack(int row, int column, int entry) { return column | (row << 7) | (entry << 11); }
__device__ __forceinline__ int bin_column(int e) { return e & 127; }
__device__ __forceinline__ int bin_row(int e) { return (e >> 7) & 15; }
__device__ __forceinline__ int bin_entry(int e) { return e >> 11; }

// ---- one F16 product C[M][N] = sum_k A B of the losses (loss_gemm.h)

enum LossEpi : int {
  LOSS_STATS = 0,  // logits: row statistics, the label's logit
  LOSS_PICK = 1,   // logits: row statistics, the logits of the teacher's tokens
  LOSS_DZ = 2,     // logits: their gradient, F16
  LOSS_DX = 3,     // dz w: fp32, added to what earlier pieces left
  LOSS_DW = 4,     // dz^T x: fp32, or codes
};

struct LossGemm {
  const void *a, *b;
  int64_t lda, ldb;       // bytes
  int b_fmt;              // of w
  int M, N, K;
  int count_is;           // the dimension that is the number of rows that count: 0 M, 1 K
  const uint32_t* hdr;
  int splits;             // parts of k, of whole groups of 128
  int v0;                 // first row of w
  // logits
  const float *factor, *lse2, *coef, *dx_factor;
  const int* label;
  float* picked2;
  const int *bins, *entries;
  int bin_columns, top;
  const int* rows;
  float* picked;
  float2* stats;
  int64_t R;
  void* dz;
  int64_t ldz;
  // gradients
  float* part;            // fp32 products, [splits][part_rows][ldp]
  int64_t ldp, part_rows;
  int accumulate;
  void* out;
  int64_t ldo;
  int out_fmt, sat, mode;
  uint32_t* amax;         // statistic of the products, or NULL
  const float *s0, *s1;   // factors of the propagated scale
};
hipError_t launch_loss_logits(const LossGemm& p, int epi, int grid, hipStream_t s);
hipError_t launch_loss_grads(const LossGemm& p, int epi, int grid, hipStream_t s);

}  // namespace scalify
