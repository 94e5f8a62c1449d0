/*
 * scalify.h - C ABI of the MI355X (gfx950) scaled-FP8 matmul library.
 *
 * Implements the hot path of Scalify's scale propagation (Balanca et al.,
 * "Scalify: scale propagation for efficient low-precision LLM training",
 * arXiv 2407.17353):
 *   - a ScaledArray is a pair (data X_d, scale X_s) with X = X_d * X_s, where
 *     X_s is a power of two held in one fp32 (Section 2; Section 3.1,
 *     Algorithm 2);
 *   - the scaled matmul propagates the output scale s_a * s_b * c with
 *     c = sqrt(K) rounded DOWN to a power of two, dividing the data by c
 *     (Section 3.2, Algorithm 3: static rule from scales and shapes under the
 *     independent-Gaussian assumption; scales rounded down);
 *   - dynamic rescaling: statistic of the data -> power of two (rounded down)
 *     -> rebalance_scale (Section 3.3, Algorithm 4); the statistic is amax;
 *   - set_scaling and get_data_and_scale (Section 3.1);
 *   - casts act on the data component only (Appendix A, cast operators);
 *   - the scaled add and activation rules, fused into the matmul epilogue
 *     (Section 3.2, Algorithm 3; Appendix C.1), and the scaled LayerNorm with
 *     the dynamic rescale of its input gradient (Appendix C.2, Section 4);
 *   - FP8 formats E4M3 / E5M2 (Section 1, Appendix A; OCP encodings on gfx950)
 *     and FP16 (E5M10) outputs.
 *
 * Conventions for every entry point
 *   - All data and scale pointers are DEVICE pointers owned by the caller.
 *     The library allocates nothing and keeps no data between calls (of a
 *     process it keeps a counter that numbers the calls, and per device the
 *     number of compute units and the address of the scratch array of
 *     scalify_matmul_noalloc); concurrent calls are safe when they use
 *     distinct workspaces. A workspace may hold anything when a call starts.
 *   - Work is enqueued on `stream` (a hipStream_t passed as void*, NULL = the
 *     default stream). No call synchronises the host or reads a scale back.
 *   - Argument errors are detected on the host before any launch; they return
 *     a status and leave every output untouched. A failed launch returns
 *     SCALIFY_ERR_HIP.
 *   - Numeric specials are not errors: NaN inputs give NaN outputs, amax
 *     ignores NaN, Inf amax or zero amax keep the propagated scale.
 *   - Preconditions not checked by the kernels: input scales are finite
 *     powers of two within the E8M0 range [2^-127, 2^127]. A NULL input scale
 *     means scale 1 (get_data_and_scale of an unscaled array, Section 3.1).
 */
#ifndef SCALIFY_H
#define SCALIFY_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    SCALIFY_OK = 0,
    SCALIFY_ERR_NULL = 1,      /* a required pointer is NULL */
    SCALIFY_ERR_DTYPE = 2,     /* unsupported data type or combination */
    SCALIFY_ERR_SHAPE = 3,     /* inconsistent or negative sizes */
    SCALIFY_ERR_LAYOUT = 4,    /* unsupported storage layout or aliasing */
    SCALIFY_ERR_ALIGN = 5,     /* data pointer or leading dimension not 16-byte aligned */
    SCALIFY_ERR_WORKSPACE = 6, /* workspace missing or too small */
    SCALIFY_ERR_VALUE = 7,     /* scalar argument out of range */
    SCALIFY_ERR_HIP = 8        /* a HIP launch failed */
} scalify_status;

typedef enum {
    SCALIFY_E4M3 = 0, /* OCP FP8 E4M3: bias 7, max 448, no Inf, NaN = S.1111.111 */
    SCALIFY_E5M2 = 1, /* OCP FP8 E5M2: bias 15, max 57344, Inf and NaN */
    SCALIFY_F16 = 2,  /* IEEE binary16 (E5M10) */
    SCALIFY_F32 = 3   /* IEEE binary32 (inputs of rescale / cast / set_scaling only) */
} scalify_dtype;

typedef enum {
    SCALIFY_RESCALE_NONE = 0,   /* static propagation rule only */
    SCALIFY_RESCALE_AMAX = 1,   /* dynamic power-of-two rescale from this call's amax */
    SCALIFY_RESCALE_DELAYED = 2 /* delayed rescale: from the amax an earlier call recorded */
} scalify_rescale_mode;

/* Activation applied by the matmul epilogue (Appendix C.1): f(x) = x * g(x)
 * with a gate g -> 0 at -inf and -> 1 at +inf; on a ScaledArray the scale
 * is kept and the data becomes X_d * g(X_d * X_s). */
typedef enum {
    SCALIFY_ACT_NONE = 0,
    SCALIFY_ACT_RELU = 1,      /* g = 1 for x > 0, else 0 */
    SCALIFY_ACT_GELU_TANH = 2, /* g = (1 + tanh(sqrt(2/pi) (x + 0.044715 x^3))) / 2 */
    SCALIFY_ACT_SILU = 3       /* g = 1 / (1 + exp(-x)) (swish) */
} scalify_activation;

/* A ScaledArray (Section 2, Section 3.1): value = decode(data) * (*scale).
 * Logical shape rows x cols.
 *   trans = 0: element (r, c) is stored at data[r * ld + c]  (ld >= cols)
 *   trans = 1: element (r, c) is stored at data[c * ld + r]  (ld >= rows)
 * The storage must hold every stored row in full: (stored rows) * ld
 * elements. `scale` points to ONE fp32 power of two on the device; NULL is
 * allowed for inputs (scale 1) and is an error for outputs. */
typedef struct {
    void* data;
    float* scale;
    int32_t dtype; /* scalify_dtype */
    int32_t trans;
    int64_t rows;
    int64_t cols;
    int64_t ld; /* in elements */
} scalify_scaled_array;

typedef struct {
    int32_t out_dtype;   /* SCALIFY_E4M3 | SCALIFY_E5M2 | SCALIFY_F16 */
    int32_t rescale;     /* scalify_rescale_mode */
    int32_t target_log2; /* t: AMAX puts the rescaled amax in [2^t, 2^(t+1)); default 0 */
    int32_t saturate;    /* 1: overflow and +-Inf -> +-max; 0: E4M3 -> NaN, E5M2/F16 -> +-Inf */
    float* acc_out;      /* optional device [M][N] fp32: the raw accumulator sum_k a_ik b_kj */
    float* amax_out;     /* optional device fp32: amax of acc * 2^-e_c over non-NaN elements
                            (with a fused add or activation: of the data the statistic is
                            gathered over, see scalify_matmul) */
    void** events;       /* optional host array of 3 hipEvent_t recorded on the stream: before
                            the GEMM kernel, after it, and after the epilogue cast (DELAYED:
                            after the amax write-back) -- timing of the fused GEMM without
                            host synchronisation; NULL = none, and a NULL entry skips
                            that record */
    const float* amax_in; /* DELAYED only (required there): device fp32 statistic recorded by
                            an earlier call (its amax_out); may be the same memory as
                            amax_out, it is read before this call writes its own */
    const scalify_scaled_array* residual; /* optional: R added to the product by the scaled
                            add rule before the activation (see scalify_matmul); E4M3, E5M2 or
                            F16, rows = M, cols = N, trans = 0, 16-byte aligned, ld a multiple
                            of 16 elements (8 for F16) and >= N, or ld = 0: one row added to
                            every row (a bias). It may be the very same matrix as out (same
                            data, dtype and ld) but must not otherwise overlap it. NULL = none */
    int32_t activation;  /* scalify_activation applied after the add; NONE = 0 */
    float* pre_out;      /* optional validation output: device fp32 [M][N], the value w the
                            rescale and cast see (after the add and the activation), whose
                            true value is w * 2^e_w (e_w as in scalify_matmul) */
    const float* a_channel_scale; /* optional channel scales of a (Section 2: a scale
                            broadcastable to the data; channel scaling): device fp32 [M],
                            one power of two (exponent in [-149, 127]) per row of the logical
                            a, i.e. per output row, on top of *a.scale; NULL = none */
    const float* b_channel_scale; /* optional: device fp32 [N], one power of two per column
                            of the logical b (per output column), on top of *b.scale,
                            16-byte aligned; NULL = none */
    const uint8_t* a_block_scale; /* optional MX block scales of a (Section 2: block
                            scaling formats such as MX as scales broadcastable to the
                            data): P, one E8M0 byte P[i][k / 32] (value 2^(byte - 127))
                            per 32 k of each row i of the logical a, scaling a[i,k] on
                            top of *a.scale, in the packed order that
                            scalify_mx_pack_block_scales writes (rows = M); device,
                            4-byte aligned; given together with b_block_scale;
                            NULL = none */
    const uint8_t* b_block_scale; /* Q, one byte Q[j][k / 32] per 32 k of each column j
                            of the logical b, packed likewise (rows = N); NULL = none */
} scalify_matmul_opts;

/* Bytes of the packed form of an MX block-scale array with `rows` rows (rows
 * of a, or columns of b) for depth K: 256 * ceil(K / 128) * ceil(rows / 64).
 * Returns 0 when rows or K is below 1. */
int64_t scalify_mx_packed_bytes(int64_t rows, int64_t K);

/* Pack MX block-scale bytes from the natural row-major order, src[r * src_ld
 * + b] for row r < rows and block b < ceil(K / 32) (src_ld >= ceil(K / 32)),
 * into the order the block-scaled matmul reads: for 128-k step t, 64-row
 * group q, k-block g in 0..3 and row r in 0..15 of the group's four 16-row
 * blocks, the 4 bytes of rows 64 q + r, + 16, + 32, + 48 at block 4 t + g
 * are the 32-bit word at byte offset ((t * ceil(rows / 64) + q) * 64 + 16 g
 * + r) * 4 of dst (lowest byte first). Blocks past ceil(K / 32) and rows
 * past `rows` are written as 127 (a factor of 1; they meet zero data).
 * dst: device, scalify_mx_packed_bytes(rows, K) bytes, 4-byte aligned,
 * not overlapping src. Pure data movement; enqueued on `stream`. Weights'
 * scales are packed once; an activation's producer can write this order
 * directly. Errors: SCALIFY_ERR_NULL (NULL src or dst with rows, K > 0),
 * SCALIFY_ERR_SHAPE (negative sizes, src_ld < ceil(K / 32), more than 2^32
 * bytes), SCALIFY_ERR_ALIGN (dst), SCALIFY_ERR_HIP. */
scalify_status scalify_mx_pack_block_scales(const uint8_t* src, int64_t rows, int64_t K,
                                            int64_t src_ld, uint8_t* dst, void* stream);

/* Exponent e_c of the matmul scale rule (Section 3.2, Algorithm 3): the
 * largest e with 2^e <= sqrt(K) (sqrt(K) rounded down to a power of two),
 * computed with integers. Returns 0 for K < 1. Host only. */
int32_t scalify_matmul_scale_log2(int64_t K);

/* Bytes of device workspace scalify_matmul needs for an M x N output with
 * the given output type and rescale mode: a 256-byte header plus, for AMAX,
 * the pre-cast intermediate (M rows of N rounded up to 16 elements; 2 bytes
 * per element for FP8 outputs, 4 for FP16). DELAYED and NONE, whose output
 * scale is known before the GEMM runs, need the header only. Returns 0 for
 * invalid arguments. */
size_t scalify_matmul_workspace_size(int64_t M, int64_t N, int32_t out_dtype, int32_t rescale);

/* Workspace bytes of a scalify_matmul call with these options: as above, but
 * an AMAX call that fuses a residual add or an activation, has channel or MX
 * block scales, or asks for pre_out, keeps an fp32 intermediate (4 bytes per
 * element for every output type).
 * Returns 0 for invalid arguments or a NULL opts. */
size_t scalify_matmul_workspace_size_opts(int64_t M, int64_t N, const scalify_matmul_opts* opts);

/* Scaled matmul on ScaledArray operands (Section 3.2, Algorithm 3; FP8
 * matmul with mixed input formats and higher-precision accumulation,
 * Appendix A), with the dynamic or delayed rescale (Section 3.3) fused:
 *   acc   = sum_k dec(a)[i,k] * dec(b)[k,j]        fp32 accumulation (MFMA)
 *   e_c   = scalify_matmul_scale_log2(K)
 *   AMAX: e_r = floor(log2 amax(acc * 2^-e_c)) - target_log2
 *         (0 when that amax is 0 or +Inf or every element is NaN)
 *   DELAYED: e_r = floor(log2 |*opts.amax_in|) - target_log2, the statistic
 *         of an earlier call (0 when it is 0, Inf or NaN); this call's amax
 *         (of acc * 2^-e_c) goes to opts.amax_out for the next call. Values
 *         the stale scale pushes past the format's range saturate (or
 *         overflow when saturate = 0). The GEMM writes the codes directly:
 *         no intermediate, no second pass over the output.
 *   NONE: e_r = 0 (the GEMM writes the codes directly, as for DELAYED)
 *   e_out = clamp(e_a + e_b + e_c + e_r, -127, 127)        (E8M0 range)
 *   out.data  = RNE(acc * 2^(e_a + e_b - e_out)) in out.dtype (saturating
 *               when opts.saturate), *out.scale = 2^e_out
 * so that dec(out) * s_out = s_a * s_b * acc up to the final rounding.
 *
 * Channel scales (opts.a_channel_scale = c, opts.b_channel_scale = d): a[i,k]
 * = dec(a)[i,k] * s_a * c[i], b[k,j] = dec(b)[k,j] * s_b * d[j]. The output
 * keeps one scalar scale: the channel factors go into the data as one
 * power-of-two product of acc (exact unless it leaves the fp32 range),
 * w = fl32(acc * c[i] * d[j]) in place of acc below (with a residual, the
 * product term is fl32(acc * 2^(e_a+e_b-e_w) * c[i] * d[j])); such a call
 * keeps an fp32 intermediate like a fused one.
 *
 * MX block scales (opts.a_block_scale = P, opts.b_block_scale = Q, both or
 * neither, each packed by scalify_mx_pack_block_scales): a[i,k] = dec(a)[i,k] * s_a * 2^(P[i][k/32] - 127), b[k,j] =
 * dec(b)[k,j] * s_b * 2^(Q[j][k/32] - 127): the matrix cores apply the block
 * factors to the products, acc = sum_k dec(a)[i,k] dec(b)[k,j]
 * 2^(P[i][k/32] + Q[j][k/32] - 254), and everything below acts on that acc
 * (the output keeps one scalar scale). The byte 0xFF (E8M0's NaN) is not a
 * scale: results of a call that uses one are unspecified. Block factors
 * that push products or partial sums out of fp32's normal range give what
 * the matrix cores give there (Inf, or subnormals and zeros). Such a call
 * keeps an fp32 intermediate; it cannot be combined with a residual, an
 * activation, pre_out or channel scales (SCALIFY_ERR_VALUE); one of the two
 * arrays alone is SCALIFY_ERR_NULL (an array of no bytes, M * K or N * K
 * zero, may be NULL), a pointer not 4-byte aligned SCALIFY_ERR_ALIGN.
 *
 * Fused scaled add and activation (opts.residual, opts.activation): the
 * epilogue first forms w, whose true value is w * 2^e_w, then rescales and
 * casts w in place of acc:
 *   no residual: w = acc, e_w = e_a + e_b, statistic over w * 2^-e_c;
 *   residual R (scale 2^q): scaled add (Algorithm 3) of the product, whose
 *     propagated scale is 2^(e_a+e_b+e_c), and R: the output scale is
 *     sqrt(s_p^2 + s_r^2) rounded down to a power of two, i.e. e_w =
 *     max(e_a + e_b + e_c, q); w = fl32(acc * 2^(e_a+e_b-e_w) + dec(R) * 2^(q-e_w))
 *     (one rounding of the sum), statistic over w;
 *   activation (Appendix C.1, after the add): w = fl32(w * g(w * 2^e_w)),
 *     scale unchanged; relu is exact, gelu and silu are evaluated in fp32
 *     (within a few ulp of the exact gate).
 *   Then e_out = clamp(e_w + (e_c, or 0 with a residual) + e_r) with e_r from
 *   the statistic of w (AMAX) or from amax_in (DELAYED), and
 *   out.data = RNE(w * 2^(e_w - e_out)); amax_out is that statistic.
 *
 * a: M x K, b: K x N, out: M x N. a and b are E4M3 or E5M2 in any mix and
 * either storage order (trans 0/1). out.trans must be 0 and out.dtype must
 * equal opts->out_dtype. All data pointers 16-byte aligned, every ld a
 * multiple of 16 elements (8 for an FP16 out). workspace: device memory of
 * at least scalify_matmul_workspace_size_opts(M, N, opts) bytes (for a call
 * with nothing fused: scalify_matmul_workspace_size(M, N, ...)), 256-byte aligned,
 * not shared with a concurrent call. Determinism: reruns are bit-identical,
 * and so are a call's accumulators in every mode. The order in which K is
 * summed depends on M, N and K: a row's accumulators may differ in their last
 * bits from those of the same row in a call of another size.
 * M, N or K may be 0 (K = 0 gives an all-zero output).
 *
 * AMAX on an output small enough that every workgroup holds its tiles (tiles
 * of 256 x 256, fewer rows or columns on smaller outputs, one per compute
 * unit; not with a fused epilogue on outputs of more than half that) runs as
 * one GEMM kernel (the single pass): its workgroups keep their output tiles in
 * registers or LDS, meet at a grid barrier on the amax statistic, and cast;
 * the output scale and amax_out are written by that kernel. Larger outputs
 * take the GEMM + cast kernel pair (faster there). The barrier's wait is bounded: if the grid is
 * not co-resident on the GPU (other work occupies its compute units), the
 * workgroups fall back to casting from the intermediate after the wait, with
 * the same result, later. Environment (read at each call):
 * SCALIFY_SINGLE_PASS=1 takes the single pass wherever it can run (any size of
 * a plain or block-scaled call, except block scales with a.trans = 1 and
 * b.trans = 0 on outputs of more than two 64 x 64 tiles per compute unit), =0
 * never;
 * SCALIFY_SPIN_TICKS=<n> sets the barrier's wait in ticks of the
 * GPU's 100 MHz counter (default 20 ms plus 4 us per 128 of K; 0 exercises
 * the fallback). SCALIFY_PERSISTENT=0 launches one workgroup per tile (and no
 * single pass) instead of the persistent grid. */
scalify_status scalify_matmul(const scalify_scaled_array* a, const scalify_scaled_array* b,
                              scalify_scaled_array* out, const scalify_matmul_opts* opts,
                              void* workspace, size_t workspace_bytes, void* stream);

/* scalify_matmul for callers that cannot allocate device memory (code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc):
 * the same computation, arguments and statuses, with the workspace taken
 * from a static array of the library instead of the caller. The library
 * holds one such array of 256 + 32 MiB bytes on every GPU it runs on, from
 * the first call with that GPU current until the process ends; this call
 * allocates nothing itself. A call whose workspace size
 * (scalify_matmul_workspace_size_opts) exceeds 256 + 32 MiB returns
 * SCALIFY_ERR_WORKSPACE and enqueues nothing: DELAYED and NONE calls fit at
 * any size (header only); AMAX calls fit while M x round_up(N, 16) x (2 for
 * FP8 outputs, 4 for FP16 outputs and fused / channel / block-scaled calls)
 * <= 32 MiB, e.g. 4096 x 4096 FP8 outputs. Every call on one GPU shares its
 * array: calls that may overlap on one GPU (other streams, other host
 * threads) race and must be ordered by the caller. `stream` must belong to
 * the current GPU. The array keeps the last call's contents; each call
 * clears what it needs cleared. SCALIFY_ERR_HIP also when the array's
 * address cannot be obtained. */
scalify_status scalify_matmul_noalloc(const scalify_scaled_array* a,
                                      const scalify_scaled_array* b, scalify_scaled_array* out,
                                      const scalify_matmul_opts* opts, void* stream);

/* Bytes of device workspace scalify_rescale needs (a 256-byte header). */
size_t scalify_rescale_workspace_size(int64_t n);

/* Dynamic rescale of a ScaledArray (Section 3.3, Algorithm 4: statistic,
 * power of two rounded down, rebalance_scale), with a cast when out.dtype
 * differs from in.dtype:
 *   AMAX: e_r = floor(log2 amax(dec(in))) - target_log2 (0 for amax 0 / +Inf /
 *         all NaN); NONE: e_r = 0
 *   e_out = clamp(e_in + e_r, -127, 127); out.data = RNE(dec(in) * 2^(e_in - e_out))
 * in.dtype: any scalify_dtype; out.dtype: E4M3, E5M2 or F16. in and out have
 * the same shape and trans and are stored contiguously (ld = cols, or rows
 * when trans = 1). out may alias in only when both have the same element
 * size; out.scale may alias in.scale. workspace >= 256 bytes. */
scalify_status scalify_rescale(const scalify_scaled_array* in, scalify_scaled_array* out,
                               int32_t mode, int32_t target_log2, int32_t saturate,
                               void* workspace, size_t workspace_bytes, void* stream);

/* Cast of the data component only; the scale is copied (Appendix A cast
 * operators): out.data = RNE(dec(in)), *out.scale = *in.scale (1 if NULL).
 * Same layout rules as scalify_rescale. */
scalify_status scalify_cast(const scalify_scaled_array* in, scalify_scaled_array* out,
                            int32_t saturate, void* stream);

/* set_scaling (Section 3.1): the output gets scale 2^new_scale_log2 and the
 * data is rescaled by the ratio of the old and new scales:
 *   out.data = RNE(dec(in) * 2^(e_in - new_scale_log2)), *out.scale = 2^new_scale_log2.
 * new_scale_log2 in [-127, 127]. out.scale must not alias in.scale. Same
 * layout rules as scalify_rescale. */
scalify_status scalify_set_scaling(const scalify_scaled_array* in, scalify_scaled_array* out,
                                   int32_t new_scale_log2, int32_t saturate, void* stream);

/* Scaled LayerNorm forward (Appendix C.2): a mean-variance normalization is
 * invariant to the scale of its input up to its eps, so it normalizes the
 * data component and gives the output scale 1. Per row r of x (R x D):
 *   mean = sum_j x_d[r,j] / D,  std = sqrt(sum_j (x_d[r,j] - mean)^2 / D),
 *   y = (x_d - mean) / (std + eps) * gamma + beta,
 *   out.data = RNE(y) in out.dtype (saturating when saturate), *out.scale = 1.
 * x.dtype: any scalify_dtype (x.scale is not read); out.dtype: E4M3, E5M2 or
 * F16. Both R x D, row-major (trans = 0), rows 16-byte aligned (ld a
 * multiple of 16 bytes, ld >= D), 1 <= D <= 8192 (any D when R = 0). gamma,
 * beta: device fp32 [D], NULL = 1 and 0. eps >= 0 (ERR_VALUE otherwise). out
 * may be the very same matrix as x (same data, element size and ld) but must
 * not otherwise overlap it. pre_out: optional device fp32 [R][D] receiving y
 * before the cast (validation). The statistics are fp32 sums in a fixed
 * order: reruns are bit-identical. Rows are read from HBM once (by the
 * backward's statistics too);
 * SCALIFY_LN_SINGLE_READ=0 (read at each call) selects the multi-pass
 * kernels instead, with the same results bit for bit. */
scalify_status scalify_layernorm_fwd(const scalify_scaled_array* x, const float* gamma,
                                     const float* beta, float eps, scalify_scaled_array* out,
                                     int32_t saturate, float* pre_out, void* stream);

/* Bytes of device workspace scalify_layernorm_bwd needs: a 256-byte header
 * plus, in fp32, 4 numbers per row and 2 x D (rounded up to 16) partial
 * parameter gradients per 32 rows (at least once). 0 for invalid sizes
 * (D > 8192). */
size_t scalify_layernorm_bwd_workspace_size(int64_t R, int64_t D);

/* Input gradient of scalify_layernorm_fwd with its dynamic rescale (the
 * LayerNorm backward rescale of the paper's experiments, Section 4, with the
 * rebalance of Section 3.3). The forward is a function of the data x_d =
 * X / X_s, so for an upstream gradient dY = dy_d * s_dy the input gradient is
 * the ScaledArray (dx, s_dy / s_x) with, per row (c = x_d - mean,
 * s = std + eps, xhat = c / s, g = dy_d * gamma):
 *   dx = (g - mean(g) - (c / std) mean(g * xhat)) / s   (last term 0 when std = 0).
 * AMAX: e_r = floor(log2 amax |dx|) - target_log2 (0 for amax 0 / Inf / all
 * NaN); NONE: e_r = 0. e_out = clamp(e(s_dy) - e(s_x) + e_r, -127, 127),
 * dx.data = RNE(dx * 2^(e(s_dy) - e(s_x) - e_out)), *dx.scale = 2^e_out.
 * dgamma[j] = sum_r dy_d[r,j] xhat[r,j] and dbeta[j] = sum_r dy_d[r,j]
 * (optional device fp32 [D]; their true values are these times s_dy);
 * amax_out: optional device fp32, the amax of |dx|; pre_out: optional device
 * fp32 [R][D], dx before the rescale (validation). dy and x: any
 * scalify_dtype, R x D with the layout rules of scalify_layernorm_fwd; dx:
 * E4M3, E5M2 or F16, the same layout, may be the very same matrix as dy or x
 * but must not otherwise overlap them. workspace: at least
 * scalify_layernorm_bwd_workspace_size(R, D) bytes, 256-byte aligned, not
 * shared with a concurrent call. Deterministic (fixed-order sums). */
scalify_status scalify_layernorm_bwd(const scalify_scaled_array* dy, const scalify_scaled_array* x,
                                     const float* gamma, float eps, scalify_scaled_array* dx,
                                     float* dgamma, float* dbeta, int32_t rescale,
                                     int32_t target_log2, int32_t saturate, float* amax_out,
                                     float* pre_out, void* workspace, size_t workspace_bytes,
                                     void* stream);

/* Scaled RMS norm forward with the residual's addition and an output in 8 bits
 * (or F16) with its scales. Per row r of x (R x D):
 *   residual R': scaled add (Section 3.2, Algorithm 3): e_h = max(e(s_x), e(s_r)),
 *     h = fl32(x_d 2^(e(s_x) - e_h) + r_d 2^(e(s_r) - e_h)); sum_out.data =
 *     RNE(h) in sum_out.dtype, *sum_out.scale = 2^e_h. With sum_out the stored
 *     (rounded) value is what the norm sees, so that scalify_rmsnorm_bwd, which
 *     reads it, is the gradient of this very function. No residual: h = x_d
 *     (x.scale is not read, as in scalify_layernorm_fwd).
 *   The normalization is scale invariant up to its eps, so the data is
 *   normalized (Appendix C.2):
 *   y = h / sqrt(sum_j h[r,j]^2 / D + eps) * gamma  (0 for a zero row, also with eps = 0)
 *   out.data = RNE(y 2^-e), *out.scale = 1, where
 *     e = 0, or, with row_scale (device fp32 [R]), e_r = clamp(floor(log2 amax_r) -
 *     target_log2, -127, 127) of the row's amax over non-NaN |y| (0 when that is 0 or
 *     Inf) and row_scale[r] = 2^e_r: the a_channel_scale of a scalify_matmul whose a
 *     is out; or, with block_scale, the same per 32 columns of a row, as E8M0 bytes
 *     e + 127 in the packed order of scalify_mx_pack_block_scales (rows = R, K = D;
 *     padding written as 127): the a_block_scale of that matmul (or, with out
 *     read through trans, its b_block_scale).
 * x.dtype: any scalify_dtype; residual, sum_out and out: E4M3, E5M2 or F16 (out
 * 8-bit with block_scale). All R x D with the layout rules of
 * scalify_layernorm_fwd, 1 <= D <= 8192 (any D when R = 0). residual, sum_out,
 * gamma (device fp32 [D], NULL = 1), row_scale, block_scale (4-byte aligned,
 * scalify_mx_packed_bytes(R, D) bytes) and pre_out (device fp32 [R][D]: y) are
 * optional (NULL). sum_out needs a residual (SCALIFY_ERR_NULL), row_scale and
 * block_scale exclude each other (SCALIFY_ERR_VALUE). out and sum_out may each be
 * the very same matrix as x or residual (same data, element size and ld) but must
 * not otherwise overlap them or each other; with a residual an output's scale
 * must not be the memory of an input's scale or the other output's
 * (SCALIFY_ERR_LAYOUT). saturate applies to both casts. Squares of F32 inputs, and
 * of sums that are not stored, of any magnitude stay in range (the row is
 * divided by a power of two first).
 * Sums are fp32 in a fixed order: reruns are bit-identical. */
scalify_status scalify_rmsnorm_fwd(const scalify_scaled_array* x,
                                   const scalify_scaled_array* residual, const float* gamma,
                                   float eps, scalify_scaled_array* sum_out,
                                   scalify_scaled_array* out, float* row_scale,
                                   uint8_t* block_scale, int32_t target_log2, int32_t saturate,
                                   float* pre_out, void* stream);

/* Bytes of device workspace scalify_rmsnorm_bwd needs: a 256-byte header plus,
 * in fp32, 4 numbers per row and up to 1024 partial rows of dgamma. 0 for
 * invalid sizes (D > 8192). */
size_t scalify_rmsnorm_bwd_workspace_size(int64_t R, int64_t D);

/* Input gradient of scalify_rmsnorm_fwd's norm with respect to the data of x,
 * the array that was normalized (sum_out, or x without a residual), plus the
 * gradient that reaches that array itself (dsum, from the residual stream),
 * with the dynamic rescale. Per row (inv = 1 / sqrt(mean(x_d^2) + eps), g =
 * dy_d * gamma):
 *   dn = inv (g - x_d inv^2 mean(g x_d)), scale s_dy / s_x
 *   dsum: scaled add: e = max(e(s_dy) - e(s_x), e(s_ds)),
 *     dx = fl32(dn 2^(e(s_dy) - e(s_x) - e) + ds_d 2^(e(s_ds) - e)); else dx = dn
 *   AMAX: e_r = floor(log2 amax |dx|) - target_log2 (0 for amax 0 / Inf / all
 *   NaN); NONE: e_r = 0. e_out = clamp(e + e_r, -127, 127), dx.data = RNE(dx
 *   2^(e - e_out)), *dx.scale = 2^e_out.
 *   dgamma[j] = sum_r dy_d[r,j] x_d[r,j] inv (optional device fp32 [D]; its true
 *   value is this times s_dy).
 * By the sum rule dx is the gradient of x and of the residual alike. dsum's
 * gradient is with respect to the sum's true value, dn's (as in
 * scalify_layernorm_bwd) to the data over its scale; both carry true values.
 * dy and x: any scalify_dtype; dsum and dx: E4M3, E5M2 or F16; all R x D with
 * the layout rules of scalify_layernorm_fwd; dx may be the very same matrix as
 * dy, x or dsum but must not otherwise overlap them, and dx.scale may be the
 * memory of an input's scale. amax_out: optional device fp32, the amax of |dx|;
 * pre_out: optional device fp32 [R][D], dx before the rescale. workspace: at
 * least scalify_rmsnorm_bwd_workspace_size(R, D) bytes, 256-byte aligned, not
 * shared with a concurrent call. Deterministic on one device (fixed-order
 * sums; their grouping depends on the device's number of compute units). */
scalify_status scalify_rmsnorm_bwd(const scalify_scaled_array* dy, const scalify_scaled_array* x,
                                   const scalify_scaled_array* dsum, const float* gamma, float eps,
                                   scalify_scaled_array* dx, float* dgamma, int32_t rescale,
                                   int32_t target_log2, int32_t saturate, float* amax_out,
                                   float* pre_out, void* workspace, size_t workspace_bytes,
                                   void* stream);

/* Attention over ScaledArrays. The matrices are those that the layer's GEMMs
 * write and read: rows are tokens, columns heads * head_dim (head h at columns h *
 * head_dim ...), any ld, so that q, k and v may be column ranges of one matrix. */
typedef struct {
    int32_t heads;       /* query heads */
    int32_t kv_heads;    /* key and value heads: heads is a multiple; query head h reads key head
                            h / (heads / kv_heads) */
    int32_t head_dim;    /* a multiple of 16 in [16, 128] */
    int32_t causal;      /* 1: query i of a sequence of L_q queries and L_k keys sees the keys
                            j <= i + L_k - L_q (the last query sees all of them) */
    int64_t batch;       /* sequences */
    float softmax_scale; /* alpha > 0, finite: the scores are alpha * q . k of the true values. Their
                            factor alpha s_q s_k log2(e) is held to [2^-100, 2^80], past which every
                            probability is that of equal scores, or of the largest alone */
    const int64_t* q_start; /* optional device [batch + 1], not decreasing: sequence b has the rows
                            q_start[b] ... q_start[b + 1] - 1 of q; NULL: rows / batch each.
                            Rows that belong to no sequence are left as they were */
    const int64_t* k_start; /* likewise the rows of k and v; NULL: rows / batch each */
    const int64_t* k_len;   /* optional device [batch]: only the first k_len[b] of sequence b's
                            rows of k and v are keys (a cache that is not full) */
    int64_t max_q;       /* with q_start: no sequence has more queries (0: any number). Rows
                            past it are left as they were, and count in L_q alone */
    int64_t max_k;       /* with k_start: no sequence has more rows of k (0: any number); the
                            backward leaves rows past it as they were. With k_len, the most
                            keys of a sequence, if that is known (0: it is not): a hint for how
                            the work is split */
} scalify_attention_opts;

/* Bytes of device workspace scalify_attention_fwd needs for rows_q rows of q and
 * rows_k rows of k. 0 where the call needs none, and for invalid arguments. */
size_t scalify_attention_fwd_workspace_size(int64_t rows_q, int64_t rows_k,
                                            const scalify_attention_opts* opts);

/* Attention forward: per sequence and query head
 *   S_ij = alpha s_q s_k sum_d q_id k_jd (admitted pairs), P = softmax_j(S), O = P v.
 * A row of P has the sum 1, so a result's data lies in the range of v's data:
 * *out.scale = *v.scale (clamped to the E8M0 range) and out.data = RNE(sum_j P_ij
 * v_jd), saturating when `saturate`. lse (optional device fp32 [heads][rows of
 * q]): log sum_j exp(S_ij), which the backward reads. A query that sees no key
 * gives zeros and lse = -Inf. What a mask or k_len hides has no effect, whatever
 * it holds (Inf, NaN); an admitted NaN gives NaN.
 * Scores, statistics and sums are fp32. The probabilities that multiply v are
 * rounded to F16 as 2^10 exp(S - m), m a running maximum of the row that a
 * later score may pass by up to 5 log 2 (half a step: 2^-11 of each; normal
 * numbers down to 2^-24 of the largest).
 * q, k, v: E4M3, E5M2 or F16, any mix of q with k and v, k and v any mix; out:
 * E4M3, E5M2 or F16. q and out: [rows of q][heads * head_dim], k and v: [rows of
 * k][kv_heads * head_dim]; trans = 0; data 16-byte aligned, every ld a multiple
 * of 16 elements (8 for F16) with 128 rows below 2^31 bytes. out must not overlap q, k
 * or v (other columns of rows of the same pitch in bytes are no overlap);
 * out.scale may be v's but not q's or k's. At most 2^30 rows, 2^30 queries times
 * heads that share a key head per sequence, and 2^31 - 1 workgroups (SCALIFY_ERR_SHAPE):
 * batch * kv_heads times one for each 32 queries and heads, and for each 128 keys, that a
 * sequence may have. Where many sequences are packed and max_q and max_k are 0, most
 * of these find no row of theirs; the two bounds spare them.
 * The values of q_start, k_start and k_len are not errors: they are clamped to
 * the matrices' rows. workspace: scalify_attention_fwd_workspace_size bytes (may be
 * NULL when that is 0), 256-byte aligned, not shared with a concurrent call.
 * Few queries, single tokens among them, take a kernel that splits the keys.
 * Deterministic: reruns are bit-identical. */
scalify_status scalify_attention_fwd(const scalify_scaled_array* q, const scalify_scaled_array* k,
                                     const scalify_scaled_array* v, scalify_scaled_array* out,
                                     float* lse, const scalify_attention_opts* opts,
                                     int32_t saturate, void* workspace, size_t workspace_bytes,
                                     void* stream);

/* Bytes of device workspace scalify_attention_bwd needs: a 256-byte header, 2
 * fp32 numbers per query row and head and 1 per key row and head, with AMAX the
 * fp32 gradients, and where the keys are too few to occupy the device, up to 16 fp32
 * copies of dk and dv that are then summed in order. 0 for invalid arguments. */
size_t scalify_attention_bwd_workspace_size(int64_t rows_q, int64_t rows_k,
                                            const scalify_attention_opts* opts, int32_t rescale);

/* Gradients of scalify_attention_fwd for the upstream gradient dO = dout, from the
 * forward's inputs and its stored results out and lse: with S as above
 *   P_ij = exp(S_ij - lse_i), delta_i = sum_d dO_id O_id, dP_ij = sum_d dO_id v_jd,
 *   dS = P (dP - delta), dV = P^T dO, dQ = alpha dS k, dK = alpha dS^T q
 * (a key head's gradients are summed over the query heads that share it), as
 * ScaledArrays with the propagated scales dv: s_do, dq: s_do s_v s_k, dk: s_do s_v
 * s_q. Each has its own rescale, as in scalify_layernorm_bwd:
 *   AMAX: e_r = floor(log2 amax of its data) - target_log2 (0 for amax 0 / Inf / all
 *   NaN), NONE: e_r = 0; e_out = clamp(propagated + e_r, -127, 127).
 * amax_out: optional device fp32 [3], the statistics of dq, dk and dv.
 * dK and dV take lse into the scores' fp32 sums, so a P is off by up to about 2^-20
 * |lse_i| of itself: F16's rounding, 2^-11, where |lse| is 2^9.
 * Rows of k past k_len get zeros. P is rounded to F16 as 2^14 P, dS to F16 times a
 * power of two that a bound of its largest magnitude among the queries and keys of a
 * workgroup, 2 max(max |dO_i| max |v_j|, max |delta_i|), gives.
 * dout, q, k, v: E4M3, E5M2 or F16; out: F16 (delta needs more than 8-bit codes
 * keep); dq, dk, dv: E4M3, E5M2 or F16. Shapes, layouts and limits as in the
 * forward; sequences must not share rows. dq, dk and dv must not overlap an
 * input or each other (other columns of rows of the same pitch are no overlap),
 * nor their scales (SCALIFY_ERR_LAYOUT). workspace: 256-byte aligned, at least
 * scalify_attention_bwd_workspace_size bytes, not shared with a concurrent call.
 * Deterministic: no sum depends on the order in which workgroups run. */
scalify_status scalify_attention_bwd(const scalify_scaled_array* dout,
                                     const scalify_scaled_array* q, const scalify_scaled_array* k,
                                     const scalify_scaled_array* v, const scalify_scaled_array* out,
                                     const float* lse, scalify_scaled_array* dq,
                                     scalify_scaled_array* dk, scalify_scaled_array* dv,
                                     const scalify_attention_opts* opts, int32_t rescale,
                                     int32_t target_log2, int32_t saturate, float* amax_out,
                                     void* workspace, size_t workspace_bytes, void* stream);

/* Human-readable name of a status code (static string). */
const char* scalify_status_string(int32_t status);

#ifdef __cplusplus
}
#endif

#endif /* SCALIFY_H */
