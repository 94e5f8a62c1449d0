// C ABI of the scaled-FP8 matmul library: argument validation on the host,
// the propagation rule table (exponent arithmetic only), workspace sizing and
// the launch sequence of each entry point. See include/scalify.h.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <stdlib.h>
#include <time.h>
#include <unistd.h>

#include <atomic>
#include <mutex>

#include "../../include/scalify.h"
#include "attention.h"
#include "gemm_choice.h"
#include "kernels.h"
#include "layernorm.h"
#include "loss.h"
#include "mid_gemm.h"
#include "rmsnorm.h"
#include "wave_gemm.h"

using namespace scalify;

namespace {

bool is_fp8(int32_t d) { return d == SCALIFY_E4M3 || d == SCALIFY_E5M2; }
bool is_out(int32_t d) { return d == SCALIFY_E4M3 || d == SCALIFY_E5M2 || d == SCALIFY_F16; }
bool is_any(int32_t d) { return d >= SCALIFY_E4M3 && d <= SCALIFY_F32; }
int64_t elem_bytes(int32_t d) { return d == SCALIFY_F32 ? 4 : (d == SCALIFY_F16 ? 2 : 1); }
bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
int64_t round_up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

constexpr int64_t kMaxDim = (int64_t)1 << 30;

// Stored rows of a matrix and the byte extent of its storage.
int64_t stored_rows(const scalify_scaled_array* x) { return x->trans ? x->cols : x->rows; }
int64_t stored_cols(const scalify_scaled_array* x) { return x->trans ? x->rows : x->cols; }

scalify_status check_matrix(const scalify_scaled_array* x, int64_t ld_multiple) {
  if (x->rows < 0 || x->cols < 0 || x->rows > kMaxDim || x->cols > kMaxDim) return SCALIFY_ERR_SHAPE;
  if (x->trans != 0 && x->trans != 1) return SCALIFY_ERR_LAYOUT;
  if (x->rows == 0 || x->cols == 0) return SCALIFY_OK;
  if (x->data == nullptr) return SCALIFY_ERR_NULL;
  if (x->ld < stored_cols(x)) return SCALIFY_ERR_SHAPE;
  if (x->ld % ld_multiple != 0 || !aligned16(x->data)) return SCALIFY_ERR_ALIGN;
  return SCALIFY_OK;
}

// fused: the call fuses a residual add or an activation, or exports pre_out;
// its intermediate is then fp32 (exact for every pre-cast value, fp32
// subnormals included).
size_t matmul_ws(int64_t M, int64_t N, int32_t out_dtype, int32_t rescale, bool fused) {
  if (M < 0 || N < 0 || !is_out(out_dtype) || rescale < SCALIFY_RESCALE_NONE ||
      rescale > SCALIFY_RESCALE_DELAYED)
    return 0;
  // DELAYED and NONE: codes written by the GEMM (the output scale is known
  // before it runs)
  if (rescale != SCALIFY_RESCALE_AMAX) return kHeaderBytes;
  const size_t bytes = (out_dtype == SCALIFY_F16 || fused) ? 4u : 2u;
  return kHeaderBytes + (size_t)M * (size_t)round_up(N, 16) * bytes;
}

// The single pass of the dynamic rescale (GEMM, grid barrier on the
// statistic, cast: one kernel) where every workgroup of the persistent grid
// holds one tile (no intermediate at all: it is faster there), the GEMM +
// cast kernel pair otherwise (the earlier tiles' intermediate, cast by the
// 4 waves of a CU after the barrier, is slower than the cast kernel).
// SCALIFY_SINGLE_PASS=1 takes the single pass wherever it can run, 0 never.
bool single_pass_choice(int64_t tiles, int grid) {
  const char* v = getenv("SCALIFY_SINGLE_PASS");
  if (v && v[0] == '1' && v[1] == 0) return true;
  if (v && v[0] == '0' && v[1] == 0) return false;
  return tiles <= grid;
}

// Where the tags of a process start: its clock, number and address layout,
// mixed (the finalizer of splitmix64, Steele, Lea and Flood 2014). Nothing here
// can fail: the callers are C.
uint64_t first_tag() noexcept {
  timespec t = {};
  clock_gettime(CLOCK_REALTIME, &t);
  uint64_t x = (uint64_t)t.tv_sec * 1000000000u + (uint64_t)t.tv_nsec;
  x ^= ((uint64_t)getpid() << 40) ^ (uint64_t)(uintptr_t)&t;
  x = (x ^ (x >> 30)) * 0xBF58476D1CE4E5B9ull;
  x = (x ^ (x >> 27)) * 0x94D049BB133111EBull;
  return x ^ (x >> 31);
}

// Tag of a call (header_tag.h): even and not zero, different for every call of
// the process, and not what a workspace holds by chance.
uint64_t next_tag() {
  static std::atomic<uint64_t> next{first_tag()};
  uint64_t t;
  do t = next.fetch_add(0x9E3779B97F4A7C15ull, std::memory_order_relaxed) << 1;
  while (t == 0);
  return t;
}

// The 4-wave kernel is persistent (one workgroup per CU walks its tiles)
// unless SCALIFY_PERSISTENT=0, which launches one workgroup per tile (and
// then no single pass, whose barrier needs the grid co-resident).
bool persistent_enabled() {
  const char* v = getenv("SCALIFY_PERSISTENT");
  return !(v && v[0] == '0' && v[1] == 0);
}

// Wait budget of the single pass's grid barrier, in ticks of the 100 MHz
// real-time counter: far beyond the arrival skew of a co-resident grid (at
// most one tile's main loop, about a microsecond per 128-deep k-step, plus
// its epilogue): 20 ms + 4 us per k-step. SCALIFY_SPIN_TICKS overrides it
// (0: a workgroup that is not the last to arrive gives up at once, which
// exercises the recovery of a grid that is not co-resident).
int64_t spin_ticks(int64_t K) {
  const char* v = getenv("SCALIFY_SPIN_TICKS");
  if (v && v[0]) return strtoll(v, nullptr, 10);
  return 2000000 + 400 * ((K + 127) / 128);
}

bool is_fused(const scalify_matmul_opts* o) {
  return o->residual != nullptr || o->activation != SCALIFY_ACT_NONE || o->pre_out != nullptr ||
         o->a_channel_scale != nullptr || o->b_channel_scale != nullptr;
}

bool has_mx(const scalify_matmul_opts* o) {
  return o->a_block_scale != nullptr || o->b_block_scale != nullptr;
}

// Calls whose pre-cast value may be any fp32 (fused epilogues, block
// scales) keep an fp32 intermediate.
bool f32_intermediate(const scalify_matmul_opts* o) { return is_fused(o) || has_mx(o); }

// Residual of the fused scaled add: M x N, row-major, ld = 0 (one row for
// every row) or ld >= N; the very same matrix as out, or disjoint from it.
scalify_status check_residual(const scalify_scaled_array* r, const scalify_scaled_array* out,
                              int64_t M, int64_t N) {
  if (!is_out(r->dtype)) return SCALIFY_ERR_DTYPE;
  if (r->rows != M || r->cols != N) return SCALIFY_ERR_SHAPE;
  if (r->trans != 0) return SCALIFY_ERR_LAYOUT;
  if (M == 0 || N == 0) return SCALIFY_OK;
  if (r->data == nullptr) return SCALIFY_ERR_NULL;
  if (r->ld != 0 && r->ld < N) return SCALIFY_ERR_SHAPE;
  if (r->ld % (r->dtype == SCALIFY_F16 ? 8 : 16) != 0 || !aligned16(r->data)) return SCALIFY_ERR_ALIGN;
  const uintptr_t r0 = (uintptr_t)r->data;
  const uintptr_t r1 = r0 + (uintptr_t)(((r->ld ? (M - 1) * r->ld : 0) + N) * elem_bytes(r->dtype));
  const uintptr_t o0 = (uintptr_t)out->data;
  const uintptr_t o1 = o0 + (uintptr_t)(((M - 1) * out->ld + N) * elem_bytes(out->dtype));
  const bool same = r->data == out->data && r->dtype == out->dtype && r->ld == out->ld;
  if (r0 < o1 && o0 < r1 && !same) return SCALIFY_ERR_LAYOUT;
  return SCALIFY_OK;
}

scalify_status check_elementwise(const scalify_scaled_array* in, const scalify_scaled_array* out) {
  if (!in || !out) return SCALIFY_ERR_NULL;
  if (!out->scale) return SCALIFY_ERR_NULL;
  if (!is_any(in->dtype) || !is_out(out->dtype)) return SCALIFY_ERR_DTYPE;
  if (in->rows < 0 || in->cols < 0 || in->rows > kMaxDim || in->cols > kMaxDim) return SCALIFY_ERR_SHAPE;
  if (in->rows != out->rows || in->cols != out->cols) return SCALIFY_ERR_SHAPE;
  if (in->trans != out->trans || (in->trans != 0 && in->trans != 1)) return SCALIFY_ERR_LAYOUT;
  const int64_t n = in->rows * in->cols;
  if (n == 0) return SCALIFY_OK;
  if (!in->data || !out->data) return SCALIFY_ERR_NULL;
  if (in->ld != stored_cols(in) || out->ld != stored_cols(out)) return SCALIFY_ERR_LAYOUT;
  if (!aligned16(in->data) || !aligned16(out->data)) return SCALIFY_ERR_ALIGN;
  // Aliasing: allowed only as the very same buffer with the same element size.
  const uintptr_t i0 = (uintptr_t)in->data, i1 = i0 + (uintptr_t)(n * elem_bytes(in->dtype));
  const uintptr_t o0 = (uintptr_t)out->data, o1 = o0 + (uintptr_t)(n * elem_bytes(out->dtype));
  if (i0 < o1 && o0 < i1 && !(i0 == o0 && elem_bytes(in->dtype) == elem_bytes(out->dtype)))
    return SCALIFY_ERR_LAYOUT;
  return SCALIFY_OK;
}

// A LayerNorm operand: R x D, row-major (trans = 0), 1 <= D <= 8192 when
// R > 0, rows 16-byte aligned (ld a multiple of 16 bytes), ld >= D.
scalify_status check_rows(const scalify_scaled_array* x, int64_t R, int64_t D) {
  if (x->rows != R || x->cols != D) return SCALIFY_ERR_SHAPE;
  if (x->trans != 0) return SCALIFY_ERR_LAYOUT;
  if (R == 0) return SCALIFY_OK;
  if (x->data == nullptr) return SCALIFY_ERR_NULL;
  if (x->ld < D) return SCALIFY_ERR_SHAPE;
  if ((x->ld * elem_bytes(x->dtype)) % 16 != 0 || !aligned16(x->data)) return SCALIFY_ERR_ALIGN;
  return SCALIFY_OK;
}

// An output may be the very same matrix as an input (same data, element
// size and ld: every row is read before it is written, by one workgroup),
// or must not overlap it.
bool rows_conflict(const scalify_scaled_array* a, const scalify_scaled_array* b, int64_t R,
                   int64_t D) {
  if (R == 0 || D == 0) return false;
  const uintptr_t a0 = (uintptr_t)a->data;
  const uintptr_t a1 = a0 + (uintptr_t)(((R - 1) * a->ld + D) * elem_bytes(a->dtype));
  const uintptr_t b0 = (uintptr_t)b->data;
  const uintptr_t b1 = b0 + (uintptr_t)(((R - 1) * b->ld + D) * elem_bytes(b->dtype));
  const bool same = a->data == b->data && elem_bytes(a->dtype) == elem_bytes(b->dtype) &&
                    a->ld == b->ld;
  return a0 < b1 && b0 < a1 && !same;
}

// ---- allocation-free matmul: its workspace is this file-scope device array
// (header + pre-cast intermediate), one copy per GPU the library runs on,
// held until the process ends. In host code `scratch` names a host-side
// stand-in; its device address, different on every GPU, comes from
// hipGetSymbolAddress with that GPU current and is the only form passed on.
constexpr size_t kNoallocScratchBytes = kHeaderBytes + ((size_t)32 << 20);
static __device__ __align__(256) uint8_t scratch[kNoallocScratchBytes];

constexpr int kMaxDevices = 64;
std::mutex g_scratch_mutex;
void* g_scratch_ptr[kMaxDevices];

// Device address of the current GPU's scratch array (looked up on the first
// call made with that GPU current, then kept).
scalify_status current_scratch(void** ptr) {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return SCALIFY_ERR_HIP;
  std::lock_guard<std::mutex> lock(g_scratch_mutex);
  if (g_scratch_ptr[dev] == nullptr) {
    void* p = nullptr;
    if (hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)) != hipSuccess || p == nullptr)
      return SCALIFY_ERR_HIP;
    g_scratch_ptr[dev] = p;
  }
  *ptr = g_scratch_ptr[dev];
  return SCALIFY_OK;
}

size_t layernorm_bwd_ws(int64_t R, int64_t D) {
  if (R < 0 || D < 0 || D > kLayerNormMaxD || R > kMaxDim) return 0;
  return kHeaderBytes + (size_t)layernorm_ws_floats(R, D) * sizeof(float);
}

size_t rmsnorm_bwd_ws(int64_t R, int64_t D) {
  if (R < 0 || D < 0 || D > kLayerNormMaxD || R > kMaxDim) return 0;
  return kHeaderBytes + (size_t)rmsnorm_ws_floats(R, D) * sizeof(float);
}

// Sizes that the losses take: places, tiles and a launch's threads are counted in 32 bits.
constexpr int64_t kMaxLoss = (int64_t)1 << 28;
bool loss_sizes_ok(int64_t R, int64_t V, int64_t D) {
  return R >= 0 && R <= kMaxLoss && V >= 1 && V <= kMaxLoss && D >= 1 && D <= ((int64_t)1 << 20) &&
         ((R + 255) / 256) * ((V + 255) / 256) <= kMaxDim && ((R + 255) / 256) * ((D + 255) / 256) <= ((int64_t)1 << 24) &&
         ((V + 255) / 256) * ((D + 255) / 256) <= kMaxDim;
}

// Two outputs of one call (different formats allowed) must not overlap at all.
bool rows_overlap(const scalify_scaled_array* a, const scalify_scaled_array* b, int64_t R, int64_t D) {
  if (R == 0 || D == 0) return false;
  const uintptr_t a0 = (uintptr_t)a->data, b0 = (uintptr_t)b->data;
  const uintptr_t a1 = a0 + (uintptr_t)(((R - 1) * a->ld + D) * elem_bytes(a->dtype));
  const uintptr_t b1 = b0 + (uintptr_t)(((R - 1) * b->ld + D) * elem_bytes(b->dtype));
  return a0 < b1 && b0 < a1;
}

// ---- attention

// Sizes of a call, from its options and the rows of q and k.
scalify_status check_attention(const scalify_attention_opts* o, int64_t rows_q, int64_t rows_k) {
  if (!o) return SCALIFY_ERR_NULL;
  if (rows_q < 0 || rows_k < 0 || rows_q > kMaxDim || rows_k > kMaxDim) return SCALIFY_ERR_SHAPE;
  if (o->heads < 1 || o->kv_heads < 1 || o->heads % o->kv_heads != 0 || o->heads > 65536) return SCALIFY_ERR_SHAPE;
  if (o->head_dim < 16 || o->head_dim > kAttnMaxD || o->head_dim % 16 != 0) return SCALIFY_ERR_SHAPE;
  if (o->batch < 1 || o->batch > kMaxDim || o->max_q < 0 || o->max_k < 0) return SCALIFY_ERR_SHAPE;
  if (!o->q_start && rows_q % o->batch != 0) return SCALIFY_ERR_SHAPE;
  if (!o->k_start && rows_k % o->batch != 0) return SCALIFY_ERR_SHAPE;
  if (o->causal != 0 && o->causal != 1) return SCALIFY_ERR_VALUE;
  if (!(o->softmax_scale > 0.0f) || !(o->softmax_scale < 3.0e38f)) return SCALIFY_ERR_VALUE;
  return SCALIFY_OK;
}

// Bounds of a sequence's rows.
int64_t most_rows(const int64_t* start, int64_t rows, int64_t batch, int64_t most) {
  if (!start) return rows / batch;
  return most > 0 && most < rows ? most : rows;
}

// The sizes a launch goes by. SCALIFY_ERR_SHAPE where a count leaves its range.
struct AttnSizes {
  int64_t max_q, max_k, keys;
  int G;
};
scalify_status attention_sizes(const scalify_attention_opts* o, int64_t rows_q, int64_t rows_k, AttnSizes* z) {
  const scalify_status st = check_attention(o, rows_q, rows_k);
  if (st != SCALIFY_OK) return st;
  z->G = o->heads / o->kv_heads;
  z->max_q = most_rows(o->q_start, rows_q, o->batch, o->max_q);
  z->max_k = most_rows(o->k_start, rows_k, o->batch, o->max_k);
  z->keys = o->k_len && o->max_k > 0 && o->max_k < z->max_k ? o->max_k : z->max_k;
  if (z->max_q * z->G > kMaxDim) return SCALIFY_ERR_SHAPE;
  // (workgroups: 32 query columns or 128 keys each; 512 and a column each where keys are split)
  const int64_t heads = o->batch * o->kv_heads;
  if (heads > 0x7FFFFFFF) return SCALIFY_ERR_SHAPE;
  const int64_t wide = heads * ((z->max_q * z->G + 31) / 32);
  const int64_t tall = heads * ((z->max_k + 127) / 128);
  if (wide > 0x7FFFFFFF || tall > 0x7FFFFFFF) return SCALIFY_ERR_SHAPE;
  return SCALIFY_OK;
}

size_t attention_fwd_ws(const scalify_attention_opts* o, int64_t rows_q, const AttnSizes& z) {
  const AttnPlan plan = attention_plan(o->batch, o->kv_heads, z.G, z.max_q, z.keys);
  if (plan.splits < 2 || rows_q == 0) return 0;
  return (size_t)plan.splits * (size_t)rows_q * (size_t)o->heads * (size_t)(o->head_dim + 2) * sizeof(float);
}

// Workspace of the backward: header, delta, norms, fp32 gradients (dk and dv of each part).
int attention_parts(const scalify_attention_opts* o, const AttnSizes& z) {
  return attention_bwd_parts(o->batch, o->kv_heads, z.G, z.max_q, z.max_k);
}

size_t attention_bwd_ws(const scalify_attention_opts* o, int64_t rows_q, int64_t rows_k, const AttnSizes& z, int32_t rescale) {
  const size_t q = (size_t)rows_q * o->heads, k = (size_t)rows_k * o->kv_heads;
  size_t n = kHeaderBytes + (size_t)round_up((int64_t)(2 * q + k), 4) * sizeof(float);
  const size_t parts = (size_t)attention_parts(o, z);
  if (rescale == SCALIFY_RESCALE_AMAX) n += q * (size_t)o->head_dim * sizeof(float);
  if (rescale == SCALIFY_RESCALE_AMAX || parts > 1) n += parts * 2 * k * (size_t)o->head_dim * sizeof(float);
  return n;
}

// A matrix of [rows][heads * head_dim].
scalify_status check_tokens(const scalify_scaled_array* x, int64_t rows, int64_t cols) {
  if (x->rows != rows || x->cols != cols) return SCALIFY_ERR_SHAPE;
  if (x->trans != 0) return SCALIFY_ERR_LAYOUT;
  if (rows == 0) return SCALIFY_OK;
  if (x->data == nullptr) return SCALIFY_ERR_NULL;
  if (x->ld < cols) return SCALIFY_ERR_SHAPE;
  if ((x->ld * elem_bytes(x->dtype)) % 16 != 0 || !aligned16(x->data)) return SCALIFY_ERR_ALIGN;
  if (x->ld >= ((int64_t)1 << 31) / 128 / elem_bytes(x->dtype)) return SCALIFY_ERR_SHAPE;
  return SCALIFY_OK;
}

// Whether two matrices share an element's memory: not if their bytes lie apart,
// or if they are other columns of rows of the same pitch.
bool tokens_overlap(const scalify_scaled_array* a, const scalify_scaled_array* b) {
  if (a->rows == 0 || b->rows == 0 || a->cols == 0 || b->cols == 0) return false;
  const uint64_t a0 = (uintptr_t)a->data, b0 = (uintptr_t)b->data;
  const uint64_t aw = (uint64_t)(a->cols * elem_bytes(a->dtype)), bw = (uint64_t)(b->cols * elem_bytes(b->dtype));
  const uint64_t ap = (uint64_t)(a->ld * elem_bytes(a->dtype)), bp = (uint64_t)(b->ld * elem_bytes(b->dtype));
  const uint64_t a1 = a0 + (uint64_t)(a->rows - 1) * ap + aw, b1 = b0 + (uint64_t)(b->rows - 1) * bp + bw;
  if (!(a0 < b1 && b0 < a1)) return false;
  if (ap != bp) return true;
  const uint64_t d = b0 >= a0 ? (b0 - a0) % ap : (ap - (a0 - b0) % ap) % ap;  // b's first column after a's
  return !(d >= aw && d + bw <= ap);
}

// Whether a contiguous vector's bytes meet those between a matrix's first and last.
bool vector_overlaps(const scalify_scaled_array* a, const void* v, int64_t bytes) {
  if (!v || bytes <= 0 || a->rows == 0 || a->cols == 0) return false;
  const uint64_t a0 = (uintptr_t)a->data, a1 = a0 + (uint64_t)(((a->rows - 1) * a->ld + a->cols) * elem_bytes(a->dtype));
  return a0 < (uintptr_t)v + (uint64_t)bytes && (uintptr_t)v < a1;
}

// ---- losses

// x [R][D], w [V][D] and the optional row scales of x; the numbers of either loss.
scalify_status check_loss(const scalify_scaled_array* x, const scalify_scaled_array* w, const float* row_scale) {
  if (!is_out(x->dtype) || !is_out(w->dtype)) return SCALIFY_ERR_DTYPE;
  const int64_t R = x->rows, V = w->rows, D = x->cols;
  if (!loss_sizes_ok(R, V, D)) return SCALIFY_ERR_SHAPE;
  scalify_status st;
  if ((st = check_tokens(x, R, D)) != SCALIFY_OK) return st;
  if ((st = check_tokens(w, V, D)) != SCALIFY_OK) return st;
  if (w->ld * elem_bytes(w->dtype) >= ((int64_t)1 << 23)) return SCALIFY_ERR_SHAPE;  // (256 rows below 2^31 bytes)
  if ((uintptr_t)row_scale & 3u) return SCALIFY_ERR_ALIGN;
  return SCALIFY_OK;
}

// The teacher's logits and tokens of a distillation.
scalify_status check_teacher(const scalify_scaled_array* t, const int64_t* index, int64_t R, float temperature) {
  if (!is_any(t->dtype)) return SCALIFY_ERR_DTYPE;
  if (t->cols < 1 || t->cols > kLossMaxTop) return SCALIFY_ERR_SHAPE;
  const scalify_status st = check_tokens(t, R, t->cols);
  if (st != SCALIFY_OK) return st;
  if (!index && R > 0) return SCALIFY_ERR_NULL;
  if ((uintptr_t)index & 7u) return SCALIFY_ERR_ALIGN;
  if (!(temperature >= 0x1p-20f) || !(temperature <= 0x1p20f)) return SCALIFY_ERR_VALUE;
  return SCALIFY_OK;
}

void loss_operands(LossParams* p, const scalify_scaled_array* x, const scalify_scaled_array* w, const float* row_scale) {
  p->x = x->data;
  p->ldx = x->ld;
  p->x_fmt = x->dtype;
  p->s_x = x->scale;
  p->w = w->data;
  p->ldw = w->ld;
  p->w_fmt = w->dtype;
  p->s_w = w->scale;
  p->row_scale = row_scale;
  p->R = (int)x->rows;
  p->V = (int)w->rows;
  p->D = (int)x->cols;
  p->temp = 1.0f;
}

void loss_teacher(LossParams* p, const scalify_scaled_array* t, const int64_t* index, float temperature) {
  p->teacher = t->data;
  p->ldt = t->ld;
  p->t_fmt = t->dtype;
  p->s_t = t->scale;
  p->top = (int)t->cols;
  p->index = index;
  p->temp = temperature;
}

scalify_status loss_forward(LossParams* p, void* workspace, size_t workspace_bytes, void* stream) {
  if (p->R == 0) return SCALIFY_OK;
  const size_t need = loss_plan(p->R, p->V, p->D, p->w_fmt, p->top, false, false, nullptr, nullptr).bytes;
  if (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255u)) return SCALIFY_ERR_WORKSPACE;
  loss_plan(p->R, p->V, p->D, p->w_fmt, p->top, false, false, p, workspace);
  return launch_loss_fwd(*p, (hipStream_t)stream) == hipSuccess ? SCALIFY_OK : SCALIFY_ERR_HIP;
}

// The backward's outputs, and the rest of its call. A piece of dw is written before the next
// one reads the operands, so no output may lie over any of them.
scalify_status loss_backward(LossParams* p, const scalify_scaled_array* x, const scalify_scaled_array* w,
                             const scalify_scaled_array* teacher, scalify_scaled_array* dx, scalify_scaled_array* dw, int32_t rescale, int32_t target_log2,
                             int32_t saturate, float* amax_out, void* workspace, size_t workspace_bytes, void* stream) {
  if (!dx && !dw) return SCALIFY_ERR_NULL;
  if ((dx && !dx->scale) || (dw && !dw->scale)) return SCALIFY_ERR_NULL;
  if ((dx && !is_out(dx->dtype)) || (dw && !is_out(dw->dtype))) return SCALIFY_ERR_DTYPE;
  if (rescale != SCALIFY_RESCALE_NONE && rescale != SCALIFY_RESCALE_AMAX) return SCALIFY_ERR_VALUE;
  if (target_log2 < -1000 || target_log2 > 1000) return SCALIFY_ERR_VALUE;
  scalify_status st;
  if (dx && (st = check_tokens(dx, p->R, p->D)) != SCALIFY_OK) return st;
  if (dw && (st = check_tokens(dw, p->V, p->D)) != SCALIFY_OK) return st;
  if (((uintptr_t)p->dloss | (uintptr_t)p->lse | (uintptr_t)p->picked | (uintptr_t)amax_out) & 3u) return SCALIFY_ERR_ALIGN;
  for (scalify_scaled_array* y : {dx, dw}) {
    if (!y) continue;
    if (tokens_overlap(y, x) || tokens_overlap(y, w)) return SCALIFY_ERR_LAYOUT;
    if (y->scale == x->scale || y->scale == w->scale || y->scale == p->s_dloss) return SCALIFY_ERR_LAYOUT;
    if (teacher && (tokens_overlap(y, teacher) || y->scale == teacher->scale)) return SCALIFY_ERR_LAYOUT;
    for (const void* v : {(const void*)p->dloss, (const void*)p->lse, (const void*)p->row_scale})
      if (vector_overlaps(y, v, 4 * (int64_t)p->R)) return SCALIFY_ERR_LAYOUT;
    const int64_t entries = (int64_t)p->R * p->top;
    if (vector_overlaps(y, p->labels, 8 * (int64_t)p->R) || vector_overlaps(y, p->index, 8 * entries) ||
        vector_overlaps(y, p->picked, 4 * entries))
      return SCALIFY_ERR_LAYOUT;
  }
  if (dx && dw && (tokens_overlap(dx, dw) || dx->scale == dw->scale)) return SCALIFY_ERR_LAYOUT;
  const bool amax = rescale == SCALIFY_RESCALE_AMAX;
  const size_t need = loss_plan(p->R, p->V, p->D, p->w_fmt, p->top, true, amax, nullptr, nullptr).bytes;
  if (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255u)) return SCALIFY_ERR_WORKSPACE;
  if (dx) {
    p->dx = dx->data;
    p->lddx = dx->ld;
    p->dx_fmt = dx->dtype;
    p->dx_scale = dx->scale;
  }
  if (dw) {
    p->dw = dw->data;
    p->lddw = dw->ld;
    p->dw_fmt = dw->dtype;
    p->dw_scale = dw->scale;
  }
  p->amax_out = amax_out;
  p->mode = amax ? 1 : 0;
  p->target = target_log2;
  p->sat = saturate != 0;
  loss_plan(p->R, p->V, p->D, p->w_fmt, p->top, true, amax, p, workspace);
  return launch_loss_bwd(*p, (hipStream_t)stream) == hipSuccess ? SCALIFY_OK : SCALIFY_ERR_HIP;
}

void attention_params(AttnParams* p, const scalify_scaled_array* q, const scalify_scaled_array* k,
                      const scalify_scaled_array* v, const scalify_attention_opts* o, const AttnSizes& z) {
  p->q = q->data;
  p->k = k->data;
  p->v = v->data;
  p->ldq = q->ld;
  p->ldk = k->ld;
  p->ldv = v->ld;
  p->q_fmt = q->dtype;
  p->k_fmt = k->dtype;
  p->v_fmt = v->dtype;
  p->s_q = q->scale;
  p->s_k = k->scale;
  p->s_v = v->scale;
  p->rows_q = q->rows;
  p->rows_k = k->rows;
  p->batch = o->batch;
  p->H = o->heads;
  p->Hkv = o->kv_heads;
  p->G = z.G;
  p->D = o->head_dim;
  p->causal = o->causal;
  p->alpha = o->softmax_scale;
  p->q_start = o->q_start;
  p->k_start = o->k_start;
  p->k_len = o->k_len;
  p->max_q = z.max_q;
  p->max_k = z.max_k;
}

}  // namespace

extern "C" {

int64_t scalify_mx_packed_bytes(int64_t rows, int64_t K) {
  if (rows < 1 || K < 1) return 0;
  return 256 * ((K + 127) / 128) * ((rows + 63) / 64);
}

scalify_status scalify_mx_pack_block_scales(const uint8_t* src, int64_t rows, int64_t K,
                                            int64_t src_ld, uint8_t* dst, void* stream) {
  if (rows < 0 || K < 0 || rows > kMaxDim || K > kMaxDim) return SCALIFY_ERR_SHAPE;
  if (rows == 0 || K == 0) return SCALIFY_OK;
  if (!src || !dst) return SCALIFY_ERR_NULL;
  if (src_ld < (K + 31) / 32 || scalify_mx_packed_bytes(rows, K) >= ((int64_t)1 << 32) ||
      rows * src_ld >= ((int64_t)1 << 32))
    return SCALIFY_ERR_SHAPE;
  if ((uintptr_t)dst & 3u) return SCALIFY_ERR_ALIGN;
  return launch_mx_pack(src, (int)rows, (int)K, (int)src_ld, dst, (hipStream_t)stream) == hipSuccess
             ? SCALIFY_OK
             : SCALIFY_ERR_HIP;
}

int32_t scalify_matmul_scale_log2(int64_t K) {
  // Largest e with 2^e <= sqrt(K), i.e. 4^e <= K (integer arithmetic only).
  int32_t e = 0;
  if (K < 1) return 0;
  while (e < 31 && ((int64_t)1 << (2 * (e + 1))) <= K) ++e;
  return e;
}

size_t scalify_matmul_workspace_size(int64_t M, int64_t N, int32_t out_dtype, int32_t rescale) {
  return matmul_ws(M, N, out_dtype, rescale, false);
}

size_t scalify_matmul_workspace_size_opts(int64_t M, int64_t N, const scalify_matmul_opts* opts) {
  if (!opts) return 0;
  return matmul_ws(M, N, opts->out_dtype, opts->rescale, f32_intermediate(opts));
}

size_t scalify_rescale_workspace_size(int64_t n) { return n < 0 ? 0 : kHeaderBytes; }

const char* scalify_status_string(int32_t s) {
  switch (s) {
    case SCALIFY_OK: return "ok";
    case SCALIFY_ERR_NULL: return "null pointer";
    case SCALIFY_ERR_DTYPE: return "unsupported dtype";
    case SCALIFY_ERR_SHAPE: return "bad shape";
    case SCALIFY_ERR_LAYOUT: return "unsupported layout or aliasing";
    case SCALIFY_ERR_ALIGN: return "misaligned pointer or leading dimension";
    case SCALIFY_ERR_WORKSPACE: return "workspace missing or too small";
    case SCALIFY_ERR_VALUE: return "scalar argument out of range";
    case SCALIFY_ERR_HIP: return "HIP launch failed";
    default: return "unknown status";
  }
}

scalify_status scalify_matmul(const scalify_scaled_array* a, const scalify_scaled_array* b,
                              scalify_scaled_array* out, const scalify_matmul_opts* opts,
                              void* workspace, size_t workspace_bytes, void* stream) {
  if (!a || !b || !out || !opts) return SCALIFY_ERR_NULL;
  if (!out->scale) return SCALIFY_ERR_NULL;
  if (!is_fp8(a->dtype) || !is_fp8(b->dtype) || !is_out(opts->out_dtype) ||
      out->dtype != opts->out_dtype)
    return SCALIFY_ERR_DTYPE;
  if (opts->rescale < SCALIFY_RESCALE_NONE || opts->rescale > SCALIFY_RESCALE_DELAYED)
    return SCALIFY_ERR_VALUE;
  if (opts->rescale == SCALIFY_RESCALE_DELAYED && !opts->amax_in) return SCALIFY_ERR_NULL;
  if (opts->target_log2 < -1000 || opts->target_log2 > 1000) return SCALIFY_ERR_VALUE;
  if (opts->activation < SCALIFY_ACT_NONE || opts->activation > SCALIFY_ACT_SILU)
    return SCALIFY_ERR_VALUE;
  if (out->trans != 0) return SCALIFY_ERR_LAYOUT;
  const int64_t M = a->rows, K = a->cols, N = b->cols;
  if (b->rows != K || out->rows != M || out->cols != N) return SCALIFY_ERR_SHAPE;
  scalify_status st;
  if ((st = check_matrix(a, 16)) != SCALIFY_OK) return st;
  if ((st = check_matrix(b, 16)) != SCALIFY_OK) return st;
  if ((st = check_matrix(out, out->dtype == SCALIFY_F16 ? 8 : 16)) != SCALIFY_OK) return st;
  const scalify_scaled_array* res = opts->residual;
  if (res && (st = check_residual(res, out, M, N)) != SCALIFY_OK) return st;
  if (!aligned16(opts->b_channel_scale) || ((uintptr_t)opts->a_channel_scale & 3u))
    return SCALIFY_ERR_ALIGN;
  const bool fused = is_fused(opts);
  const bool mx = has_mx(opts);
  const int64_t mx_a_bytes = scalify_mx_packed_bytes(M, K), mx_b_bytes = scalify_mx_packed_bytes(N, K);
  if (mx) {
    // an array of no bytes (M, N or K zero) may be NULL
    if ((!opts->a_block_scale && M * K > 0) || (!opts->b_block_scale && N * K > 0))
      return SCALIFY_ERR_NULL;
    if (fused) return SCALIFY_ERR_VALUE;
    if (((uintptr_t)opts->a_block_scale | (uintptr_t)opts->b_block_scale) & 3u)
      return SCALIFY_ERR_ALIGN;
    if (mx_a_bytes >= ((int64_t)1 << 32) || mx_b_bytes >= ((int64_t)1 << 32)) return SCALIFY_ERR_SHAPE;
  }
  // 32-bit byte offsets inside the GEMM kernel, including the range-checked
  // reads of up to one tile past the last stored row.
  if (M && K && (stored_rows(a) + 256) * a->ld + 256 >= ((int64_t)1 << 32)) return SCALIFY_ERR_SHAPE;
  if (K && N && (stored_rows(b) + 256) * b->ld + 256 >= ((int64_t)1 << 32)) return SCALIFY_ERR_SHAPE;
  const size_t need = matmul_ws(M, N, opts->out_dtype, opts->rescale, fused || mx);
  if (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255u))
    return SCALIFY_ERR_WORKSPACE;

  hipStream_t s = (hipStream_t)stream;
  uint32_t* hdr = (uint32_t*)workspace;
  const int e_c = scalify_matmul_scale_log2(K);
  const bool amax_mode = opts->rescale == SCALIFY_RESCALE_AMAX;
  const bool delayed = opts->rescale == SCALIFY_RESCALE_DELAYED;
  // Delayed or no rescale: the output scale is known before the GEMM runs
  // (from the statistic of an earlier call, or the propagated scale itself),
  // so the GEMM casts straight to codes (no intermediate). Dynamic rescale:
  // the GEMM writes a pre-cast intermediate: 16-bit for FP8 outputs of the
  // plain epilogue, fp32 for FP16 outputs, for fused epilogues and with
  // block scales (whose accumulators may be fp32 subnormals, which the
  // 16-bit encoding does not keep exactly); the single pass keeps each
  // workgroup's last tile out of it and casts in the same kernel.
  const int epi = !amax_mode ? EPI_DIRECT
                             : ((opts->out_dtype == SCALIFY_F16 || fused || mx) ? EPI_INTER32
                                                                                 : EPI_INTER16);
  // (256 x 256 kernel without the single pass: fused, or block scales of
  // A [K][M] with B [K][N])
  const bool tn_mx = mx && a->trans != 0 && b->trans == 0;
  const bool persistent = persistent_enabled();
  const int cus = gemm4_grid(1 << 30);
  // The direct cast needs the header only for a statistic, or where the
  // output scale shares memory with what other workgroups still read.
  const float* o = out->scale;
  const bool counted = !amax_mode && (opts->amax_out || o == a->scale || o == b->scale ||
                                      (res && o == res->scale) || (delayed && o == opts->amax_in));
  const GemmChoice gc = gemm_choice(M, N, K, cus, fused, mx, amax_mode, amax_mode || counted);
  int grid = (int)gc.tiles;
  if (persistent && gc.kind != GEMM_FUSED && grid > gc.resident * cus) grid = gc.resident * cus;
  // Single pass where each workgroup can hold its tiles: the wave kernel by
  // its choice always, the others with one tile each. (Forced, the 256 x 256
  // kernel holds its last tile and passes the others through the intermediate.)
  const bool single_pass =
      amax_mode && persistent && gc.kind != GEMM_FUSED &&
      (gc.kind == GEMM_BIG ? !tn_mx && single_pass_choice(gc.tiles, grid)
                           : (gc.kind == GEMM_WAVE || gc.tiles <= grid) && single_pass_choice(0, 0));
  // Exponent offset of the statistic: the matmul data is acc * 2^-e_c; with
  // a residual the statistic is taken over w itself.
  const int e_cc = res ? 0 : e_c;
  hipEvent_t* ev = (hipEvent_t*)opts->events;
  auto record = [&](int i) {
    return !ev || !ev[i] || hipEventRecord(ev[i], s) == hipSuccess;
  };

  if (M == 0 || N == 0) {
    EmptyMatmul q = {};
    q.s0 = a->scale;
    q.s1 = b->scale;
    q.s_res = res ? res->scale : nullptr;
    q.residual = res ? 1 : 0;
    q.e_c = e_c;
    q.amax_in = delayed ? opts->amax_in : nullptr;
    q.target = opts->target_log2;
    q.out_scale = out->scale;
    q.amax_out = opts->amax_out;
    if (!record(0) || launch_empty_matmul(q, s) != hipSuccess || !record(1) || !record(2))
      return SCALIFY_ERR_HIP;
    return SCALIFY_OK;
  }

  GemmParams p = {};
  p.a = (const uint8_t*)a->data;
  p.b = (const uint8_t*)b->data;
  p.lda = a->ld;
  p.ldb = b->ld;
  p.M = (int)M;
  p.N = (int)N;
  p.K = (int)K;
  p.tiles_m = (int)((M + gc.tm - 1) / gc.tm);
  p.tiles_n = (int)((N + gc.tn - 1) / gc.tn);
  p.a_bytes = (uint32_t)(stored_rows(a) * a->ld);
  p.b_bytes = (uint32_t)(stored_rows(b) * b->ld);
  p.e_c = e_c;
  p.e_cc = e_cc;
  p.s0 = a->scale;
  p.s1 = b->scale;
  p.s_res = res ? res->scale : nullptr;
  p.amax_in = delayed ? opts->amax_in : nullptr;
  p.residual = res ? 1 : 0;
  p.counted = counted;
  p.uses_header = epi != EPI_DIRECT || p.counted;
  p.tag = p.uses_header ? next_tag() : 0;
  p.sat = opts->saturate != 0;
  p.hdr = hdr;
  p.inter = (uint8_t*)workspace + kHeaderBytes;
  p.ldw = round_up(N, 16);
  p.acc_out = opts->acc_out;
  p.out = out->data;
  p.ldc = out->ld;
  p.out_fmt = opts->out_dtype;
  p.res = res ? res->data : nullptr;
  p.ldr = res ? res->ld : 0;
  p.res_fmt = res ? res->dtype : 0;
  p.act = opts->activation;
  p.pre_out = opts->pre_out;
  p.ch_a = opts->a_channel_scale;
  p.ch_b = opts->b_channel_scale;
  // (the block-scale kernels run whenever the product has terms: K > 0)
  p.mx_a = mx && K > 0 ? opts->a_block_scale : nullptr;
  p.mx_b = mx && K > 0 ? opts->b_block_scale : nullptr;
  p.mx_groups_a = (int)((M + 63) / 64);
  p.mx_groups_b = (int)((N + 63) / 64);
  p.mx_a_bytes = (uint32_t)mx_a_bytes;
  p.mx_b_bytes = (uint32_t)mx_b_bytes;
  p.grid = grid;
  p.epi = epi;
  p.single_pass = single_pass ? 1 : 0;
  p.target = opts->target_log2;
  p.out_scale = out->scale;
  p.amax_out = opts->amax_out;
  p.spin_ticks = spin_ticks(K);
  const bool ta = a->trans != 0, tb = b->trans != 0;
  if (!record(0)) return SCALIFY_ERR_HIP;
  if ((gc.kind == GEMM_WAVE  ? launch_wave_gemm(p, ta, tb, a->dtype, b->dtype, s)
       : gc.kind == GEMM_MID ? launch_mid_gemm(p, ta, tb, a->dtype, b->dtype, gc.mid, s)
       : gc.kind == GEMM_FUSED ? launch_fused_gemm(p, ta, tb, a->dtype, b->dtype, s)
                             : launch_gemm(p, ta, tb, a->dtype, b->dtype, s)) != hipSuccess)
    return SCALIFY_ERR_HIP;
  if (!record(1)) return SCALIFY_ERR_HIP;
  if (epi != EPI_DIRECT && !single_pass) {
    // Second pass of the two-kernel dynamic rescale: global amax -> rescale
    // exponent -> output scale, and the cast of the intermediate.
    EpilogueParams q = {};
    q.inter = p.inter;
    q.ldw = p.ldw;
    q.out = out->data;
    q.ldc = out->ld;
    q.M = (int)M;
    q.N = (int)N;
    q.e_c = e_cc;
    q.target = opts->target_log2;
    q.sat = p.sat;
    q.mode = 1;
    q.hdr = hdr;
    q.out_scale = out->scale;
    q.amax_out = opts->amax_out;
    if (launch_epilogue_cast(q, epi == EPI_INTER32, opts->out_dtype, s) != hipSuccess)
      return SCALIFY_ERR_HIP;
  }
  return record(2) ? SCALIFY_OK : SCALIFY_ERR_HIP;
}

scalify_status scalify_matmul_noalloc(const scalify_scaled_array* a,
                                      const scalify_scaled_array* b, scalify_scaled_array* out,
                                      const scalify_matmul_opts* opts, void* stream) {
  if (!a || !b || !out || !opts) return SCALIFY_ERR_NULL;
  // A workspace larger than the array is refused before anything is enqueued
  // (scalify_matmul checks the other arguments first and returns their error).
  void* ws = nullptr;
  const scalify_status st = current_scratch(&ws);
  if (st != SCALIFY_OK) return st;
  return scalify_matmul(a, b, out, opts, ws, kNoallocScratchBytes, stream);
}

scalify_status scalify_rescale(const scalify_scaled_array* in, scalify_scaled_array* out,
                               int32_t mode, int32_t target_log2, int32_t saturate,
                               void* workspace, size_t workspace_bytes, void* stream) {
  scalify_status st = check_elementwise(in, out);
  if (st != SCALIFY_OK) return st;
  if (mode != SCALIFY_RESCALE_NONE && mode != SCALIFY_RESCALE_AMAX) return SCALIFY_ERR_VALUE;
  if (target_log2 < -1000 || target_log2 > 1000) return SCALIFY_ERR_VALUE;
  if (!workspace || workspace_bytes < kHeaderBytes || ((uintptr_t)workspace & 255u))
    return SCALIFY_ERR_WORKSPACE;
  hipStream_t s = (hipStream_t)stream;
  uint32_t* hdr = (uint32_t*)workspace;
  const int64_t n = in->rows * in->cols;
  // The statistic's kernel keeps the header itself; without one, a header is
  // needed only for a snapshot of an input scale that the output scale overwrites.
  const bool stat = mode == SCALIFY_RESCALE_AMAX && n > 0;
  const bool snapshot = stat || in->scale == out->scale;
  if (stat) {
    if (launch_amax(in->data, in->dtype, n, in->scale, hdr, next_tag(), s) != hipSuccess)
      return SCALIFY_ERR_HIP;
  } else if (snapshot) {
    if (launch_prologue(hdr, in->scale, s) != hipSuccess) return SCALIFY_ERR_HIP;
  }
  ElemParams p = {};
  p.in = in->data;
  p.out = out->data;
  p.n = n;
  p.rule = stat ? RULE_AMAX : RULE_KEEP;
  p.target = target_log2;
  p.sat = saturate != 0;
  p.hdr = snapshot ? hdr : nullptr;
  p.in_scale = in->scale;
  p.out_scale = out->scale;
  if (launch_elementwise(p, in->dtype, out->dtype, s) != hipSuccess) return SCALIFY_ERR_HIP;
  return SCALIFY_OK;
}

scalify_status scalify_cast(const scalify_scaled_array* in, scalify_scaled_array* out,
                            int32_t saturate, void* stream) {
  scalify_status st = check_elementwise(in, out);
  if (st != SCALIFY_OK) return st;
  ElemParams p = {};
  p.in = in->data;
  p.out = out->data;
  p.n = in->rows * in->cols;
  p.rule = RULE_COPY;
  p.sat = saturate != 0;
  p.in_scale = in->scale;
  p.out_scale = out->scale;
  if (launch_elementwise(p, in->dtype, out->dtype, (hipStream_t)stream) != hipSuccess)
    return SCALIFY_ERR_HIP;
  return SCALIFY_OK;
}

scalify_status scalify_set_scaling(const scalify_scaled_array* in, scalify_scaled_array* out,
                                   int32_t new_scale_log2, int32_t saturate, void* stream) {
  scalify_status st = check_elementwise(in, out);
  if (st != SCALIFY_OK) return st;
  if (new_scale_log2 < -127 || new_scale_log2 > 127) return SCALIFY_ERR_VALUE;
  if (in->scale != nullptr && in->scale == out->scale) return SCALIFY_ERR_LAYOUT;
  ElemParams p = {};
  p.in = in->data;
  p.out = out->data;
  p.n = in->rows * in->cols;
  p.rule = RULE_FIXED;
  p.e_fixed = new_scale_log2;
  p.sat = saturate != 0;
  p.in_scale = in->scale;
  p.out_scale = out->scale;
  if (launch_elementwise(p, in->dtype, out->dtype, (hipStream_t)stream) != hipSuccess)
    return SCALIFY_ERR_HIP;
  return SCALIFY_OK;
}

scalify_status scalify_layernorm_fwd(const scalify_scaled_array* x, const float* gamma,
                                     const float* beta, float eps, scalify_scaled_array* out,
                                     int32_t saturate, float* pre_out, void* stream) {
  if (!x || !out) return SCALIFY_ERR_NULL;
  if (!out->scale) return SCALIFY_ERR_NULL;
  if (!is_any(x->dtype) || !is_out(out->dtype)) return SCALIFY_ERR_DTYPE;
  const int64_t R = x->rows, D = x->cols;
  if (R < 0 || D < 0 || R > kMaxDim) return SCALIFY_ERR_SHAPE;
  if (R > 0 && (D < 1 || D > kLayerNormMaxD)) return SCALIFY_ERR_SHAPE;
  if (!(eps >= 0.0f) || !(eps < 3.0e38f)) return SCALIFY_ERR_VALUE;
  if (!aligned16(gamma) || !aligned16(beta) || !aligned16(pre_out)) return SCALIFY_ERR_ALIGN;
  scalify_status st;
  if ((st = check_rows(x, R, D)) != SCALIFY_OK) return st;
  if ((st = check_rows(out, R, D)) != SCALIFY_OK) return st;
  if (rows_conflict(x, out, R, D)) return SCALIFY_ERR_LAYOUT;
  LnParams p = {};
  p.x = x->data;
  p.ldx = x->ld;
  p.x_fmt = x->dtype;
  p.gamma = gamma;
  p.beta = beta;
  p.out = out->data;
  p.ldo = out->ld;
  p.pre_out = pre_out;
  p.R = R;
  p.D = (int)D;
  p.eps = eps;
  p.sat = saturate != 0;
  p.out_scale = out->scale;
  if (launch_layernorm_fwd(p, out->dtype, (hipStream_t)stream) != hipSuccess)
    return SCALIFY_ERR_HIP;
  return SCALIFY_OK;
}

size_t scalify_layernorm_bwd_workspace_size(int64_t R, int64_t D) { return layernorm_bwd_ws(R, D); }

scalify_status scalify_layernorm_bwd(const scalify_scaled_array* dy, const scalify_scaled_array* x,
                                     const float* gamma, float eps, scalify_scaled_array* dx,
                                     float* dgamma, float* dbeta, int32_t rescale,
                                     int32_t target_log2, int32_t saturate, float* amax_out,
                                     float* pre_out, void* workspace, size_t workspace_bytes,
                                     void* stream) {
  if (!dy || !x || !dx) return SCALIFY_ERR_NULL;
  if (!dx->scale) return SCALIFY_ERR_NULL;
  if (!is_any(dy->dtype) || !is_any(x->dtype) || !is_out(dx->dtype)) return SCALIFY_ERR_DTYPE;
  if (rescale != SCALIFY_RESCALE_NONE && rescale != SCALIFY_RESCALE_AMAX) return SCALIFY_ERR_VALUE;
  if (target_log2 < -1000 || target_log2 > 1000) return SCALIFY_ERR_VALUE;
  if (!(eps >= 0.0f) || !(eps < 3.0e38f)) return SCALIFY_ERR_VALUE;
  const int64_t R = x->rows, D = x->cols;
  if (R < 0 || D < 0 || R > kMaxDim) return SCALIFY_ERR_SHAPE;
  if (R > 0 && (D < 1 || D > kLayerNormMaxD)) return SCALIFY_ERR_SHAPE;
  if (!aligned16(gamma) || !aligned16(dgamma) || !aligned16(dbeta) || !aligned16(pre_out))
    return SCALIFY_ERR_ALIGN;
  scalify_status st;
  if ((st = check_rows(x, R, D)) != SCALIFY_OK) return st;
  if ((st = check_rows(dy, R, D)) != SCALIFY_OK) return st;
  if ((st = check_rows(dx, R, D)) != SCALIFY_OK) return st;
  if (rows_conflict(dx, dy, R, D) || rows_conflict(dx, x, R, D)) return SCALIFY_ERR_LAYOUT;
  const size_t need = layernorm_bwd_ws(R, D);
  if (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255u))
    return SCALIFY_ERR_WORKSPACE;
  LnParams p = {};
  p.x = x->data;
  p.ldx = x->ld;
  p.x_fmt = x->dtype;
  p.dy = dy->data;
  p.lddy = dy->ld;
  p.dy_fmt = dy->dtype;
  p.gamma = gamma;
  p.out = dx->data;
  p.ldo = dx->ld;
  p.pre_out = pre_out;
  p.R = R;
  p.D = (int)D;
  p.eps = eps;
  p.sat = saturate != 0;
  p.target = target_log2;
  p.mode = rescale == SCALIFY_RESCALE_AMAX ? 1 : 0;
  p.hdr = (uint32_t*)workspace;
  p.tag = next_tag();
  p.s_dy = dy->scale;
  p.s_x = x->scale;
  p.partial = (float*)((uint8_t*)workspace + kHeaderBytes);
  p.out_scale = dx->scale;
  p.amax_out = amax_out;
  p.dgamma = dgamma;
  p.dbeta = dbeta;
  if (launch_layernorm_bwd(p, dx->dtype, (hipStream_t)stream) != hipSuccess)
    return SCALIFY_ERR_HIP;
  return SCALIFY_OK;
}

scalify_status scalify_rmsnorm_fwd(const scalify_scaled_array* x,
                                   const scalify_scaled_array* residual, const float* gamma,
                                   float eps, scalify_scaled_array* sum_out,
                                   scalify_scaled_array* out, float* row_scale,
                                   uint8_t* block_scale, int32_t target_log2, int32_t saturate,
                                   float* pre_out, void* stream) {
  if (!x || !out || !out->scale) return SCALIFY_ERR_NULL;
  if (sum_out && (!residual || !sum_out->scale)) return SCALIFY_ERR_NULL;
  if (!is_any(x->dtype) || !is_out(out->dtype) || (residual && !is_out(residual->dtype)) ||
      (sum_out && !is_out(sum_out->dtype)) || (block_scale && !is_fp8(out->dtype)))
    return SCALIFY_ERR_DTYPE;
  if (row_scale && block_scale) return SCALIFY_ERR_VALUE;
  if (target_log2 < -1000 || target_log2 > 1000) return SCALIFY_ERR_VALUE;
  if (!(eps >= 0.0f) || !(eps < 3.0e38f)) return SCALIFY_ERR_VALUE;
  const int64_t R = x->rows, D = x->cols;
  if (R < 0 || D < 0 || R > kMaxDim) return SCALIFY_ERR_SHAPE;
  if (R > 0 && (D < 1 || D > kLayerNormMaxD)) return SCALIFY_ERR_SHAPE;
  if (!aligned16(gamma) || !aligned16(pre_out)) return SCALIFY_ERR_ALIGN;
  if (((uintptr_t)row_scale & 3u) || ((uintptr_t)block_scale & 3u)) return SCALIFY_ERR_ALIGN;
  scalify_status st;
  if ((st = check_rows(x, R, D)) != SCALIFY_OK) return st;
  if ((st = check_rows(out, R, D)) != SCALIFY_OK) return st;
  if (rows_conflict(x, out, R, D)) return SCALIFY_ERR_LAYOUT;
  if (residual) {
    if ((st = check_rows(residual, R, D)) != SCALIFY_OK) return st;
    if (rows_conflict(residual, out, R, D)) return SCALIFY_ERR_LAYOUT;
    if (out->scale == x->scale || out->scale == residual->scale) return SCALIFY_ERR_LAYOUT;
  }
  if (sum_out) {
    if ((st = check_rows(sum_out, R, D)) != SCALIFY_OK) return st;
    if (rows_conflict(x, sum_out, R, D) || rows_conflict(residual, sum_out, R, D) ||
        rows_overlap(out, sum_out, R, D))
      return SCALIFY_ERR_LAYOUT;
    if (sum_out->scale == x->scale || sum_out->scale == residual->scale || sum_out->scale == out->scale)
      return SCALIFY_ERR_LAYOUT;
  }
  RmsParams p = {};
  p.x = x->data;
  p.ldx = x->ld;
  p.x_fmt = x->dtype;
  p.s_x = x->scale;
  p.has_res = residual != nullptr;
  if (residual) {
    p.res = residual->data;
    p.ldr = residual->ld;
    p.res_fmt = residual->dtype;
    p.s_res = residual->scale;
  }
  p.gamma = gamma;
  if (sum_out) {
    p.sum = sum_out->data;
    p.lds = sum_out->ld;
    p.sum_fmt = sum_out->dtype;
    p.sum_scale = sum_out->scale;
  }
  p.out = out->data;
  p.ldo = out->ld;
  p.out_fmt = out->dtype;
  p.out_scale = out->scale;
  p.row_scale = row_scale;
  p.block_scale = block_scale;
  p.pre_out = pre_out;
  p.R = R;
  p.D = (int)D;
  p.eps = eps;
  p.sat = saturate != 0;
  p.target = target_log2;
  return launch_rmsnorm_fwd(p, (hipStream_t)stream) == hipSuccess ? SCALIFY_OK : SCALIFY_ERR_HIP;
}

size_t scalify_rmsnorm_bwd_workspace_size(int64_t R, int64_t D) { return rmsnorm_bwd_ws(R, D); }

scalify_status scalify_rmsnorm_bwd(const scalify_scaled_array* dy, const scalify_scaled_array* x,
                                   const scalify_scaled_array* dsum, const float* gamma, float eps,
                                   scalify_scaled_array* dx, float* dgamma, int32_t rescale,
                                   int32_t target_log2, int32_t saturate, float* amax_out,
                                   float* pre_out, void* workspace, size_t workspace_bytes,
                                   void* stream) {
  if (!dy || !x || !dx || !dx->scale) return SCALIFY_ERR_NULL;
  if (!is_any(dy->dtype) || !is_any(x->dtype) || !is_out(dx->dtype) || (dsum && !is_out(dsum->dtype)))
    return SCALIFY_ERR_DTYPE;
  if (rescale != SCALIFY_RESCALE_NONE && rescale != SCALIFY_RESCALE_AMAX) return SCALIFY_ERR_VALUE;
  if (target_log2 < -1000 || target_log2 > 1000) return SCALIFY_ERR_VALUE;
  if (!(eps >= 0.0f) || !(eps < 3.0e38f)) return SCALIFY_ERR_VALUE;
  const int64_t R = x->rows, D = x->cols;
  if (R < 0 || D < 0 || R > kMaxDim) return SCALIFY_ERR_SHAPE;
  if (D > kLayerNormMaxD || (R > 0 && D < 1)) return SCALIFY_ERR_SHAPE;
  if (!aligned16(gamma) || !aligned16(dgamma) || !aligned16(pre_out)) return SCALIFY_ERR_ALIGN;
  scalify_status st;
  if ((st = check_rows(x, R, D)) != SCALIFY_OK) return st;
  if ((st = check_rows(dy, R, D)) != SCALIFY_OK) return st;
  if ((st = check_rows(dx, R, D)) != SCALIFY_OK) return st;
  if (rows_conflict(dx, dy, R, D) || rows_conflict(dx, x, R, D)) return SCALIFY_ERR_LAYOUT;
  if (dsum) {
    if ((st = check_rows(dsum, R, D)) != SCALIFY_OK) return st;
    if (rows_conflict(dx, dsum, R, D)) return SCALIFY_ERR_LAYOUT;
  }
  const size_t need = rmsnorm_bwd_ws(R, D);
  if (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255u))
    return SCALIFY_ERR_WORKSPACE;
  RmsParams p = {};
  p.x = x->data;
  p.ldx = x->ld;
  p.x_fmt = x->dtype;
  p.s_x = x->scale;
  p.dy = dy->data;
  p.lddy = dy->ld;
  p.dy_fmt = dy->dtype;
  p.s_dy = dy->scale;
  p.has_res = dsum != nullptr;
  if (dsum) {
    p.res = dsum->data;
    p.ldr = dsum->ld;
    p.res_fmt = dsum->dtype;
    p.s_res = dsum->scale;
  }
  p.gamma = gamma;
  p.out = dx->data;
  p.ldo = dx->ld;
  p.out_fmt = dx->dtype;
  p.out_scale = dx->scale;
  p.pre_out = pre_out;
  p.R = R;
  p.D = (int)D;
  p.eps = eps;
  p.sat = saturate != 0;
  p.target = target_log2;
  p.mode = rescale == SCALIFY_RESCALE_AMAX ? 1 : 0;
  p.hdr = (uint32_t*)workspace;
  p.tag = next_tag();
  p.partial = (float*)((uint8_t*)workspace + kHeaderBytes);
  p.amax_out = amax_out;
  p.dgamma = dgamma;
  return launch_rmsnorm_bwd(p, (hipStream_t)stream) == hipSuccess ? SCALIFY_OK : SCALIFY_ERR_HIP;
}

size_t scalify_attention_fwd_workspace_size(int64_t rows_q, int64_t rows_k,
                                            const scalify_attention_opts* opts) {
  AttnSizes z;
  if (attention_sizes(opts, rows_q, rows_k, &z) != SCALIFY_OK) return 0;
  return attention_fwd_ws(opts, rows_q, z);
}

scalify_status scalify_attention_fwd(const scalify_scaled_array* q, const scalify_scaled_array* k,
                                     const scalify_scaled_array* v, scalify_scaled_array* out,
                                     float* lse, const scalify_attention_opts* opts,
                                     int32_t saturate, void* workspace, size_t workspace_bytes,
                                     void* stream) {
  if (!q || !k || !v || !out || !opts || !out->scale) return SCALIFY_ERR_NULL;
  if (!is_out(q->dtype) || !is_out(k->dtype) || !is_out(v->dtype) || !is_out(out->dtype))
    return SCALIFY_ERR_DTYPE;
  AttnSizes z;
  scalify_status st = attention_sizes(opts, q->rows, k->rows, &z);
  if (st != SCALIFY_OK) return st;
  const int64_t cq = (int64_t)opts->heads * opts->head_dim, ck = (int64_t)opts->kv_heads * opts->head_dim;
  if ((st = check_tokens(q, q->rows, cq)) != SCALIFY_OK) return st;
  if ((st = check_tokens(k, k->rows, ck)) != SCALIFY_OK) return st;
  if ((st = check_tokens(v, k->rows, ck)) != SCALIFY_OK) return st;
  if ((st = check_tokens(out, q->rows, cq)) != SCALIFY_OK) return st;
  if (((uintptr_t)lse & 3u) != 0) return SCALIFY_ERR_ALIGN;
  if (((uintptr_t)opts->q_start | (uintptr_t)opts->k_start | (uintptr_t)opts->k_len) & 7u) return SCALIFY_ERR_ALIGN;
  if (tokens_overlap(out, q) || tokens_overlap(out, k) || tokens_overlap(out, v)) return SCALIFY_ERR_LAYOUT;
  if (out->scale == q->scale || out->scale == k->scale) return SCALIFY_ERR_LAYOUT;
  const size_t need = attention_fwd_ws(opts, q->rows, z);
  if (need > 0 && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255u)))
    return SCALIFY_ERR_WORKSPACE;
  const AttnPlan plan = attention_plan(opts->batch, opts->kv_heads, z.G, z.max_q, z.keys);
  AttnParams p = {};
  attention_params(&p, q, k, v, opts, z);
  p.out = out->data;
  p.ldo = out->ld;
  p.out_fmt = out->dtype;
  p.out_scale = out->scale;
  p.lse = lse;
  p.sat = saturate != 0;
  p.splits = plan.splits;
  p.part_o = (float*)workspace;
  p.part_ml = (float2*)((float*)workspace + (size_t)plan.splits * (size_t)q->rows * (size_t)cq);
  return launch_attention_fwd(p, plan, (hipStream_t)stream) == hipSuccess ? SCALIFY_OK : SCALIFY_ERR_HIP;
}

size_t scalify_attention_bwd_workspace_size(int64_t rows_q, int64_t rows_k,
                                            const scalify_attention_opts* opts, int32_t rescale) {
  AttnSizes z;
  if (attention_sizes(opts, rows_q, rows_k, &z) != SCALIFY_OK) return 0;
  if (rescale != SCALIFY_RESCALE_NONE && rescale != SCALIFY_RESCALE_AMAX) return 0;
  return attention_bwd_ws(opts, rows_q, rows_k, z, rescale);
}

scalify_status scalify_attention_bwd(const scalify_scaled_array* dout,
                                     const scalify_scaled_array* q, const scalify_scaled_array* k,
                                     const scalify_scaled_array* v, const scalify_scaled_array* out,
                                     const float* lse, scalify_scaled_array* dq,
                                     scalify_scaled_array* dk, scalify_scaled_array* dv,
                                     const scalify_attention_opts* opts, int32_t rescale,
                                     int32_t target_log2, int32_t saturate, float* amax_out,
                                     void* workspace, size_t workspace_bytes, void* stream) {
  if (!dout || !q || !k || !v || !out || !dq || !dk || !dv || !opts) return SCALIFY_ERR_NULL;
  if (!dq->scale || !dk->scale || !dv->scale) return SCALIFY_ERR_NULL;
  const scalify_scaled_array* const in[5] = {dout, q, k, v, out};
  scalify_scaled_array* const grad[3] = {dq, dk, dv};
  for (const scalify_scaled_array* x : in)
    if (!is_out(x->dtype)) return SCALIFY_ERR_DTYPE;
  for (const scalify_scaled_array* x : grad)
    if (!is_out(x->dtype)) return SCALIFY_ERR_DTYPE;
  if (out->dtype != SCALIFY_F16) return SCALIFY_ERR_DTYPE;
  if (rescale != SCALIFY_RESCALE_NONE && rescale != SCALIFY_RESCALE_AMAX) return SCALIFY_ERR_VALUE;
  if (target_log2 < -1000 || target_log2 > 1000) return SCALIFY_ERR_VALUE;
  AttnSizes z;
  scalify_status st = attention_sizes(opts, q->rows, k->rows, &z);
  if (st != SCALIFY_OK) return st;
  const int64_t cq = (int64_t)opts->heads * opts->head_dim, ck = (int64_t)opts->kv_heads * opts->head_dim;
  // workgroups of the row statistics (16 rows of a head) and of the casts (4 rows)
  if ((q->rows * opts->heads + k->rows * opts->kv_heads) / 16 > 0x7FFFFFF0 ||
      opts->batch * (((z.max_q > z.max_k ? z.max_q : z.max_k) + 3) / 4) > 0x7FFFFFFF)
    return SCALIFY_ERR_SHAPE;
  for (const scalify_scaled_array* x : {dout, q, (const scalify_scaled_array*)out, (const scalify_scaled_array*)dq})
    if ((st = check_tokens(x, q->rows, cq)) != SCALIFY_OK) return st;
  for (const scalify_scaled_array* x : {k, v, (const scalify_scaled_array*)dk, (const scalify_scaled_array*)dv})
    if ((st = check_tokens(x, k->rows, ck)) != SCALIFY_OK) return st;
  if (!lse && q->rows > 0) return SCALIFY_ERR_NULL;
  if (((uintptr_t)lse & 3u) != 0) return SCALIFY_ERR_ALIGN;
  if (((uintptr_t)opts->q_start | (uintptr_t)opts->k_start | (uintptr_t)opts->k_len) & 7u) return SCALIFY_ERR_ALIGN;
  for (int i = 0; i < 3; ++i) {
    for (const scalify_scaled_array* x : in)
      if (tokens_overlap(grad[i], x) || grad[i]->scale == x->scale) return SCALIFY_ERR_LAYOUT;
    for (int j = 0; j < i; ++j)
      if (tokens_overlap(grad[i], grad[j]) || grad[i]->scale == grad[j]->scale) return SCALIFY_ERR_LAYOUT;
  }
  const size_t need = attention_bwd_ws(opts, q->rows, k->rows, z, rescale);
  if (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255u)) return SCALIFY_ERR_WORKSPACE;
  AttnParams p = {};
  attention_params(&p, q, k, v, opts, z);
  p.out = out->data;
  p.ldo = out->ld;
  p.out_fmt = out->dtype;
  p.out_scale = out->scale;
  p.lse = (float*)lse;
  p.sat = saturate != 0;
  p.dout = dout->data;
  p.lddo = dout->ld;
  p.do_fmt = dout->dtype;
  p.s_do = dout->scale;
  const size_t nq = (size_t)q->rows * opts->heads, nk = (size_t)k->rows * opts->kv_heads;
  p.amax = (uint32_t*)workspace;
  p.delta = (float*)((uint8_t*)workspace + kHeaderBytes);
  p.nd2 = p.delta + nq;
  p.nv2 = p.nd2 + nq;
  p.parts = attention_parts(opts, z);
  p.part = p.delta + round_up((int64_t)(2 * nq + nk), 4);
  if (rescale == SCALIFY_RESCALE_AMAX) {
    p.dq32 = p.part;
    p.dk32 = p.part = p.dq32 + nq * (size_t)opts->head_dim;
    p.dv32 = p.dk32 + nk * (size_t)opts->head_dim;
  }
  p.dq = dq->data;
  p.dk = dk->data;
  p.dv = dv->data;
  p.lddq = dq->ld;
  p.lddk = dk->ld;
  p.lddv = dv->ld;
  p.dq_fmt = dq->dtype;
  p.dk_fmt = dk->dtype;
  p.dv_fmt = dv->dtype;
  p.dq_scale = dq->scale;
  p.dk_scale = dk->scale;
  p.dv_scale = dv->scale;
  p.amax_out = amax_out;
  p.mode = rescale == SCALIFY_RESCALE_AMAX ? 1 : 0;
  p.target = target_log2;
  return launch_attention_bwd(p, (hipStream_t)stream) == hipSuccess ? SCALIFY_OK : SCALIFY_ERR_HIP;
}

size_t scalify_cross_entropy_fwd_workspace_size(int64_t R, int64_t V, int64_t D, int32_t w_dtype) {
  if (!loss_sizes_ok(R, V, D) || !is_out(w_dtype)) return 0;
  return loss_plan(R, V, D, w_dtype, 0, false, false, nullptr, nullptr).bytes;
}

scalify_status scalify_cross_entropy_fwd(const scalify_scaled_array* x, const scalify_scaled_array* w,
                                         const int64_t* labels, const float* row_scale, float* loss,
                                         float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  if (!x || !w) return SCALIFY_ERR_NULL;
  const scalify_status st = check_loss(x, w, row_scale);
  if (st != SCALIFY_OK) return st;
  if (x->rows > 0 && (!labels || !loss)) return SCALIFY_ERR_NULL;
  if (((uintptr_t)labels & 7u) || (((uintptr_t)loss | (uintptr_t)lse) & 3u)) return SCALIFY_ERR_ALIGN;
  LossParams p = {};
  loss_operands(&p, x, w, row_scale);
  p.labels = labels;
  p.loss = loss;
  p.lse = lse;
  return loss_forward(&p, workspace, workspace_bytes, stream);
}

size_t scalify_cross_entropy_bwd_workspace_size(int64_t R, int64_t V, int64_t D, int32_t w_dtype, int32_t rescale) {
  if (!loss_sizes_ok(R, V, D) || !is_out(w_dtype)) return 0;
  if (rescale != SCALIFY_RESCALE_NONE && rescale != SCALIFY_RESCALE_AMAX) return 0;
  return loss_plan(R, V, D, w_dtype, 0, true, rescale == SCALIFY_RESCALE_AMAX, nullptr, nullptr).bytes;
}

scalify_status scalify_cross_entropy_bwd(const float* dloss, const float* dloss_scale,
                                         const scalify_scaled_array* x, const scalify_scaled_array* w,
                                         const int64_t* labels, const float* row_scale, const float* lse,
                                         scalify_scaled_array* dx, scalify_scaled_array* dw, int32_t rescale,
                                         int32_t target_log2, int32_t saturate, float* amax_out,
                                         void* workspace, size_t workspace_bytes, void* stream) {
  if (!x || !w) return SCALIFY_ERR_NULL;
  const scalify_status st = check_loss(x, w, row_scale);
  if (st != SCALIFY_OK) return st;
  if (x->rows > 0 && (!labels || !lse)) return SCALIFY_ERR_NULL;
  if ((uintptr_t)labels & 7u) return SCALIFY_ERR_ALIGN;
  LossParams p = {};
  loss_operands(&p, x, w, row_scale);
  p.dloss = dloss;
  p.s_dloss = dloss_scale;
  p.labels = labels;
  p.lse = (float*)lse;
  return loss_backward(&p, x, w, nullptr, dx, dw, rescale, target_log2, saturate, amax_out, workspace, workspace_bytes, stream);
}

size_t scalify_distillation_fwd_workspace_size(int64_t R, int64_t V, int64_t D, int64_t top, int32_t w_dtype) {
  if (!loss_sizes_ok(R, V, D) || !is_out(w_dtype) || top < 1 || top > kLossMaxTop) return 0;
  return loss_plan(R, V, D, w_dtype, (int)top, false, false, nullptr, nullptr).bytes;
}

scalify_status scalify_distillation_fwd(const scalify_scaled_array* x, const scalify_scaled_array* w,
                                        const scalify_scaled_array* teacher, const int64_t* index,
                                        float temperature, const float* row_scale, float* loss, float* lse,
                                        float* picked, void* workspace, size_t workspace_bytes, void* stream) {
  if (!x || !w || !teacher) return SCALIFY_ERR_NULL;
  scalify_status st = check_loss(x, w, row_scale);
  if (st != SCALIFY_OK) return st;
  if ((st = check_teacher(teacher, index, x->rows, temperature)) != SCALIFY_OK) return st;
  if (x->rows > 0 && !loss) return SCALIFY_ERR_NULL;
  if (((uintptr_t)loss | (uintptr_t)lse | (uintptr_t)picked) & 3u) return SCALIFY_ERR_ALIGN;
  LossParams p = {};
  loss_operands(&p, x, w, row_scale);
  loss_teacher(&p, teacher, index, temperature);
  p.loss = loss;
  p.lse = lse;
  p.picked = picked;
  return loss_forward(&p, workspace, workspace_bytes, stream);
}

size_t scalify_distillation_bwd_workspace_size(int64_t R, int64_t V, int64_t D, int64_t top, int32_t w_dtype,
                                               int32_t rescale) {
  if (!loss_sizes_ok(R, V, D) || !is_out(w_dtype) || top < 1 || top > kLossMaxTop) return 0;
  if (rescale != SCALIFY_RESCALE_NONE && rescale != SCALIFY_RESCALE_AMAX) return 0;
  return loss_plan(R, V, D, w_dtype, (int)top, true, rescale == SCALIFY_RESCALE_AMAX, nullptr, nullptr).bytes;
}

scalify_status scalify_distillation_bwd(const float* dloss, const float* dloss_scale,
                                        const scalify_scaled_array* x, const scalify_scaled_array* w,
                                        const scalify_scaled_array* teacher, const int64_t* index,
                                        float temperature, const float* row_scale, const float* lse,
                                        const float* picked, scalify_scaled_array* dx, scalify_scaled_array* dw,
                                        int32_t rescale, int32_t target_log2, int32_t saturate, float* amax_out,
                                        void* workspace, size_t workspace_bytes, void* stream) {
  if (!x || !w || !teacher) return SCALIFY_ERR_NULL;
  scalify_status st = check_loss(x, w, row_scale);
  if (st != SCALIFY_OK) return st;
  if ((st = check_teacher(teacher, index, x->rows, temperature)) != SCALIFY_OK) return st;
  if (x->rows > 0 && (!lse || !picked)) return SCALIFY_ERR_NULL;
  LossParams p = {};
  loss_operands(&p, x, w, row_scale);
  loss_teacher(&p, teacher, index, temperature);
  p.dloss = dloss;
  p.s_dloss = dloss_scale;
  p.lse = (float*)lse;
  p.picked = (float*)picked;
  return loss_backward(&p, x, w, teacher, dx, dw, rescale, target_log2, saturate, amax_out, workspace, workspace_bytes, stream);
}

}  // extern "C"
