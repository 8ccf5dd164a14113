/*
 * nm.h -- C ABI of the MI355X (gfx950) NeuralMatrix inference library.
 *
 * The library computes transformer encoder layers (and residual CNNs, as convolutions in matrix
 * form) with linear matrix operations only (paper, Section 3): every linear operator is an
 * int8 x int8 -> int32 matrix product (Section 3.1) and
 * every nonlinear operator (GELU, the exponential and the reciprocal of softmax, the reciprocal
 * square root of LayerNorm) is a piecewise-linear table y = k[s]*x + b[s] whose segment s is found
 * by quantising x (Section 3.2, Post-Training Approximation; Algorithm 3 for k, b; Algorithm 2
 * for merged segments).  The last section adds a decoder's step over a paged key-value cache.
 *
 * Conventions
 *   - Plain C.  Every function returns an nm_status (0 = NM_OK, negative = error) unless stated.
 *     After an error nm_last_error() returns a thread-local description.
 *   - "device" pointers are HIP device memory owned by the caller; "host" pointers are ordinary
 *     memory.  The library allocates only nm_tables objects.  Compute entry points are
 *     asynchronous on the given stream (a hipStream_t passed as void*, NULL = default stream),
 *     allocate nothing and never synchronise with the host.
 *   - Arguments are validated before the first HIP call; validation failures leave the GPU
 *     untouched (and work on a machine without a GPU).
 *   - Matrices are row-major.  Activations are [rows, cols]; weights are [N, K] with K contiguous
 *     (the layout of a fully connected layer's weight, and the one the int8 matrix cores want for
 *     both operands).  Attention tensors are [B, S, heads, d] viewed as [B*S, H]; a head is a
 *     column slice, nothing is transposed in memory by the caller.
 *   - Floating-point work is IEEE binary32, round-to-nearest-even, in one normative operation
 *     order, so that segment indices and int8 codes are reproducible bit for bit:
 *       segment:   u = (x - lo) * inv_w  (one subtract, one multiply), clamped in float to
 *                  [0, nseg-1], floor.  A break point belongs to the segment on its right;
 *                  x >= hi uses the last segment, x < lo and NaN the first (inputs outside the
 *                  range share the edge segments' parameters).
 *       PWL:       y = fma(k[s], x, b[s])
 *       int8 code: q = clamp(rint(v * inv_scale), -127, 127)
 *       row sum:   element j goes to accumulator (j / 4) % 64; each accumulator adds its elements
 *                  in increasing j starting from +0; the 64 partial sums are combined by a
 *                  butterfly with partner masks 32, 16, 8, 4, 2, 1.
 */
#ifndef NM_H
#define NM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    NM_OK = 0,
    NM_ERR_INVALID_ARG = -1, /* null pointer, non-positive dimension, hi <= lo, nseg < 1, ... */
    NM_ERR_UNSUPPORTED = -2, /* a shape the kernels do not cover (limits are stated per call) */
    NM_ERR_ALLOC = -3,
    NM_ERR_HIP = -4,         /* a HIP runtime call failed; see nm_last_error() */
    NM_ERR_WORKSPACE = -5    /* workspace too small or misaligned */
} nm_status;

/* Nonlinear functions a table can be built for (the paper's four: e^x, sqrt x, 1/x, GELU, plus
 * the reciprocal square root LayerNorm uses here, ReLU which is already piecewise linear, and the
 * identity). */
enum { NM_FUNC_GELU = 0, NM_FUNC_EXP = 1, NM_FUNC_RECIP = 2, NM_FUNC_RSQRT = 3, NM_FUNC_RELU = 4,
       NM_FUNC_SQRT = 5, NM_FUNC_IDENTITY = 6 };

enum {
    NM_TABLE_CLAMP_INPUT = 1,  /* clamp x to [lo, hi] before evaluation instead of extrapolating */
    NM_TABLE_BIAS_CORRECT = 2, /* Algorithm 3: shift b by the expectation bias when |dE| > e_th */
    NM_TABLE_MERGE = 4,        /* Algorithm 2: merge neighbouring primary segments whose slope
                                  stays within dk_th of the slope at the last kept start point;
                                  nseg is then the number of primary cells */
    NM_TABLE_COMPACT = 8       /* keep a merged table in two levels as well: one {k, b} per merged
                                  segment plus one byte per primary cell naming its segment (at most
                                  256 segments), so that a kernel holds n_segments * 8 + nseg bytes of
                                  it instead of nseg * 8.  nm_pwl_apply looks such a table up in two
                                  steps (cell of x, segment of the cell), and so does nm_gemm_pwl
                                  where it writes more than int8 codes or has a residual, per-column
                                  output scales or a table that clamps; everything else uses the
                                  expanded form, one look-up instead of two.  Results are identical
                                  either way; reported segment indices are always primary cell indices */
};

/* Types of a tensor.  The calls on int8 codes take I32 and F32; those of a decode step (the last section) say which of the others. */
enum { NM_DT_I32 = 0, NM_DT_F32 = 1, NM_DT_BF16 = 2, NM_DT_F16 = 3, NM_DT_I8 = 4 };

#define NM_MAX_SEGMENTS 4096 /* per table */
#define NM_MAX_TABLES 16     /* per nm_tables object */

typedef struct {
    int32_t func;  /* NM_FUNC_* */
    float lo;      /* range of the approximated input; hi > lo */
    float hi;
    int32_t nseg;  /* number of uniform segments (cells), 1 .. NM_MAX_SEGMENTS */
    int32_t flags; /* NM_TABLE_* */
    float e_th;    /* Algorithm 3 threshold (0 = always correct) */
    float dk_th;   /* Algorithm 2 slope threshold (used with NM_TABLE_MERGE) */
} nm_table_desc;

typedef struct nm_tables nm_tables; /* opaque: host copy + device blob of up to 16 tables */

/* Thread-local text of the last error on this thread ("" if none). Never NULL. */
const char* nm_last_error(void);

/* Library version, major * 1000 + minor. */
int32_t nm_version(void);

/*
 * Host-only table construction (Section 3.2: fixed-length segments, each fitted by the line
 * through the function values at its two ends, so neighbouring lines meet; Algorithm 3 step 1;
 * with NM_TABLE_BIAS_CORRECT the rest of Algorithm 3; with NM_TABLE_MERGE Algorithm 2 first and
 * the chords are taken over the merged segments, expanded back onto the nseg primary cells).
 * All arithmetic in binary64, results rounded once to binary32.
 * k, b: host arrays of desc->nseg floats (written).  inv_w: host, receives (float)(nseg/(hi-lo)).
 * n_distinct (may be NULL): number of distinct (k, b) pairs = segments after merging.
 * Never touches the GPU.
 */
int32_t nm_table_build_host(const nm_table_desc* desc, float* k, float* b, float* inv_w,
                            int32_t* n_distinct);

/*
 * Build n tables on the host (as nm_table_build_host) and upload them as one device blob on
 * `stream`.  descs: host array of n descriptors, 1 <= n <= NM_MAX_TABLES.  *out receives a new
 * object owned by the caller (nm_tables_destroy).  This is an offline call: it waits for the
 * upload on `stream` before it returns, so the tables may be used from any stream afterwards.
 */
int32_t nm_build_tables(const nm_table_desc* descs, int32_t n, void* stream, nm_tables** out);

/*
 * Same, but k and b come from the caller: k[i], b[i] are host arrays of descs[i].nseg floats.
 * descs[i].func / e_th / dk_th are ignored, lo / hi / nseg / NM_TABLE_CLAMP_INPUT /
 * NM_TABLE_COMPACT are used (the two-level form is derived from runs of equal {k, b}).
 */
int32_t nm_tables_from_arrays(const nm_table_desc* descs, int32_t n, const float* const* k,
                              const float* const* b, void* stream, nm_tables** out);

/* Number of tables in the object (0 for NULL). */
int32_t nm_tables_count(const nm_tables* t);

/*
 * Read table idx back from the host copy.  Any of desc, k_host, b_host, inv_w may be NULL.
 * k_host, b_host: host arrays of nseg floats.
 */
int32_t nm_tables_get(const nm_tables* t, int32_t idx, nm_table_desc* desc, float* k_host,
                      float* b_host, float* inv_w);

/*
 * The two-level form of table idx (built with NM_TABLE_COMPACT): number of merged segments, the
 * segment of every primary cell (host array of nseg bytes), and the segments' parameters (host
 * arrays of *n_segments floats; query the count first).  Any output may be NULL.
 */
int32_t nm_tables_get_compact(const nm_tables* t, int32_t idx, int32_t* n_segments, uint8_t* cell_to_segment,
                              float* k_host, float* b_host);

/* Frees the host copy and the device blob.  NULL is allowed.  The caller must make sure no kernel
 * that uses the tables is still running. */
void nm_tables_destroy(nm_tables* t);

/* ---------------------------------------------------------------------------------------------
 * nm_gemm_pwl: int8 GEMM with the fused epilogue (Section 3.1: a fully connected layer is a
 * matrix multiplication, a residual connection a matrix addition; Section 3.2 for the table).
 *
 *   acc[m,n] = sum_k A[m,k] * W[n,k]                      exact, int32
 *   v = fma((float)acc, alpha_n, bias_n)                   alpha_n = alpha_vec ? alpha_vec[n] : alpha
 *   v = fma((float)resid[m,n], resid_scale, v)             if resid
 *   v = PWL_table(v)                                       if table_idx >= 0
 *   out_f32[m,n] = v;  out_q[m,n] = int8 code of v with out_inv_scale_n;  out_acc[m,n] = acc;
 *   dbg_seg[m,n] = segment index of v (only written when a table is given)
 *
 * All pointers are device pointers; A [M,K], W [N,K], resid / outputs [M,N], all contiguous.
 * bias, alpha_vec, out_inv_scale_vec: [N] or NULL.  Any output may be NULL (at least one is
 * required).  Limits: 1 <= M, N, K; K <= 65536 (so |acc| <= K * 127^2 < 2^31); M*N < 2^31.
 * Shapes whose K is a multiple of 16 with 16-byte aligned A and W take the fast loader; any
 * other shape is computed by a slower loader with identical results.
 * Debug switches (environment, read once per process; results never change, only the kernel that
 * computes them): NM_GEMM_GENERIC=1 sends every product whose operand is not gathered from an image to the
 * generic kernel; NM_GEMM_CFG=big|wide|split|small|mid3|mid2|oldbig|direct<0-6>|unaligned<0-3>|relu<2,5-11>|
 * tile<0-9> forces a kernel and its tile configuration where that one's requirements hold (anywhere else, and
 * where the value is not one of these, the rules choose as without it); NM_ATTN_UNFUSED=1 keeps
 * nm_encoder_layer's attention on the three separate kernels.
 * --------------------------------------------------------------------------------------------- */
typedef struct {
    int32_t M, N, K;
    const int8_t* A;
    const int8_t* W;
    const float* bias;
    const float* alpha_vec;
    float alpha;
    const int8_t* resid;
    float resid_scale;
    const nm_tables* tables;
    int32_t table_idx; /* -1 = no nonlinearity */
    float out_inv_scale;
    const float* out_inv_scale_vec;
    int8_t* out_q;
    float* out_f32;
    int32_t* out_acc;
    uint16_t* dbg_seg;
    /* split_cols > 0: the int8 code of column n uses out_inv_scale3[min(n / split_cols, 2)] instead of
     * out_inv_scale (a fused Q | K | V projection has one output scale per third); out_inv_scale_vec
     * must then be NULL.  0: not used. */
    int32_t split_cols;
    float out_inv_scale3[3];
} nm_gemm_desc;

int32_t nm_gemm_pwl(const nm_gemm_desc* desc, void* stream);

/* ---------------------------------------------------------------------------------------------
 * nm_softmax_pwl: row softmax with PWL exponential and PWL reciprocal (the paper lists e^x and
 * 1/x among the functions it approximates; the decomposition is this library's):
 *   m = max_j in_j;  t_j = (float)(in_j - m) * alpha;  e_j = PWL_exp(t_j);
 *   S = canonical row sum of e;  r = PWL_recip(S);  p_j = e_j * r.
 * in: device [rows, cols] int32 (NM_DT_I32; the subtraction is then exact) or fp32 (NM_DT_F32).
 * Outputs (device, any may be NULL, at least one of out_q / out_f32 required): out_q int8 codes
 * of p with out_inv_scale, out_f32 p, dbg_seg_exp [rows, cols] exp segment of every element,
 * dbg_seg_recip [rows] reciprocal segment of every row.
 * Limits: 1 <= cols <= 4096, rows >= 0, rows * cols < 2^40; alpha finite (NM_ERR_INVALID_ARG).
 * --------------------------------------------------------------------------------------------- */
int32_t nm_softmax_pwl(const void* in, int32_t in_dtype, float alpha, int64_t rows, int32_t cols,
                       const nm_tables* tables, int32_t exp_idx, int32_t recip_idx,
                       float out_inv_scale, int8_t* out_q, float* out_f32, uint16_t* dbg_seg_exp,
                       uint16_t* dbg_seg_recip, void* stream);

/* ---------------------------------------------------------------------------------------------
 * nm_layernorm_pwl: row LayerNorm with a PWL reciprocal square root:
 *   mu = rowsum(x) * inv_L;  d_j = x_j - mu;  var = rowsum_fma(d_j * d_j) * inv_L;
 *   r = PWL_rsqrt(var + eps);  y_j = fma(d_j * r, gamma_j, beta_j);   inv_L = (float)(1.0 / cols)
 * in: device fp32 [rows, cols]; gamma, beta: device fp32 [cols].
 * Outputs (device, any may be NULL, at least one of out_q / out_f32 required): out_q int8 codes of
 * y with out_inv_scale, out_f32 y, dbg_seg [rows] the rsqrt segment of every row.
 * Limits: 1 <= cols <= 4096, rows >= 0.
 * --------------------------------------------------------------------------------------------- */
int32_t nm_layernorm_pwl(const float* in, const float* gamma, const float* beta, float eps,
                         int64_t rows, int32_t cols, const nm_tables* tables, int32_t rsqrt_idx,
                         float out_inv_scale, int8_t* out_q, float* out_f32, uint16_t* dbg_seg,
                         void* stream);

/*
 * nm_layernorm_pwl2: the same with the two functions the paper's list names instead of one rsqrt
 * table: sd = PWL_sqrt(var + eps); r = PWL_recip(sd).  dbg_seg_sqrt / dbg_seg_recip: [rows].
 */
int32_t nm_layernorm_pwl2(const float* in, const float* gamma, const float* beta, float eps,
                          int64_t rows, int32_t cols, const nm_tables* tables, int32_t sqrt_idx,
                          int32_t recip_idx, float out_inv_scale, int8_t* out_q, float* out_f32,
                          uint16_t* dbg_seg_sqrt, uint16_t* dbg_seg_recip, void* stream);

/* ---------------------------------------------------------------------------------------------
 * nm_pwl_apply: the stand-alone element-wise PWL calculation over a flat buffer (Section 3: an
 * operator that is piecewise linear is evaluated by finding each element's segment, gathering k
 * and b, and one multiply-add):  x = (float)in_i * alpha;  y = PWL(x).
 * in: device int32 or fp32 [n].  Outputs (device, any may be NULL, at least one required):
 * out_q int8, out_f32, dbg_seg uint16.  n >= 0.
 * --------------------------------------------------------------------------------------------- */
int32_t nm_pwl_apply(const void* in, int32_t in_dtype, float alpha, int64_t n,
                     const nm_tables* tables, int32_t idx, float out_inv_scale, int8_t* out_q,
                     float* out_f32, uint16_t* dbg_seg, void* stream);

/* ---------------------------------------------------------------------------------------------
 * Attention products (Section 3.1: attention is a linear operation mapped to matrix products).
 * qkv: device int8 [B*S, 3H]: columns [0,H) queries, [H,2H) keys, [2H,3H) values; head t owns
 * columns t*d .. t*d+d-1 of each third, d = H / heads.
 *   nm_attn_scores :  scores[b,t,i,j] = sum_c Q[b,i,t,c] * K[b,j,t,c]       int32 [B,heads,S,S]
 *   nm_attn_context:  acc = sum_j P[b,t,i,j] * V[b,j,t,c];  v = fma((float)acc, alpha, 0);
 *                     ctx[b,i,t*d+c] = int8 code of v with out_inv_scale      int8 [B*S, H]
 * p: device int8 [B,heads,S,S].  Limits: H % heads == 0, S <= 4096.
 * --------------------------------------------------------------------------------------------- */
int32_t nm_attn_scores(const int8_t* qkv, int32_t B, int32_t S, int32_t H, int32_t heads,
                       int32_t* scores, void* stream);
int32_t nm_attn_context(const int8_t* p, const int8_t* qkv, int32_t B, int32_t S, int32_t H,
                        int32_t heads, float alpha, float out_inv_scale, int8_t* ctx,
                        void* stream);

/* ---------------------------------------------------------------------------------------------
 * nm_attention_pwl: the three attention steps in one kernel (scores, softmax-PWL, context), with
 * results bit-identical to nm_attn_scores -> nm_softmax_pwl -> nm_attn_context; the int32 scores
 * and the int8 probabilities stay in registers.  scores_out / p_out (device, [B,heads,S,S]) may be
 * NULL; when given they receive the intermediate tensors.
 * Limits: head size H / heads == 64, S <= 512, qkv 16-byte aligned, H % 16 == 0; other shapes
 * return NM_ERR_UNSUPPORTED and the caller uses the three separate calls.  alpha_scores must be
 * finite (NM_ERR_INVALID_ARG otherwise).
 * --------------------------------------------------------------------------------------------- */
int32_t nm_attention_pwl(const int8_t* qkv, int32_t B, int32_t S, int32_t H, int32_t heads,
                         float alpha_scores, const nm_tables* tables, int32_t exp_idx,
                         int32_t recip_idx, float inv_s_p, float alpha_ctx, float inv_s_ctx,
                         int8_t* ctx, int32_t* scores_out, int8_t* p_out, void* stream);

/* ---------------------------------------------------------------------------------------------
 * nm_encoder_layer: one post-LayerNorm (BERT ordering) encoder layer, no mask, no dropout:
 *   1 QKV projection (+bias), each third requantised with its own scale
 *   2 scores = Q K^T per (batch, head)                        int32
 *   3 softmax-PWL over each score row                          int8
 *   4 context = P V per (batch, head), requantised             int8
 *   5 output projection + bias + residual(x)                   fp32
 *   6 LayerNorm-PWL                                            int8
 *   7 FFN1 + bias, GELU-PWL in the GEMM epilogue               int8
 *   8 FFN2 + bias + residual(LN1 output)                       fp32
 *   9 LayerNorm-PWL                                            int8 (+ fp32)
 * All weight / vector pointers are device pointers.  The float multipliers are formed by the
 * caller from the tensors' quantisation scales (s_*) and passed as binary32 numbers.
 * --------------------------------------------------------------------------------------------- */
typedef struct {
    int32_t B, S, H, heads, F;
    const int8_t* Wqkv; const float* bqkv; /* [3H, H] rows Wq | Wk | Wv; [3H] */
    const int8_t* Wo;   const float* bo;   /* [H, H]; [H] */
    const int8_t* W1;   const float* b1;   /* [F, H]; [F] */
    const int8_t* W2;   const float* b2;   /* [H, F]; [H] */
    const float* gamma1; const float* beta1; /* [H] */
    const float* gamma2; const float* beta2; /* [H] */
    float eps1, eps2;
    float alpha_qkv;              /* s_x * s_wqkv */
    float inv_s_q, inv_s_k, inv_s_v;
    float alpha_scores;           /* s_q * s_k / sqrt(d) */
    float inv_s_p;
    float alpha_ctx;              /* s_p * s_v */
    float inv_s_ctx;
    float alpha_o;                /* s_ctx * s_wo */
    float resid1_scale;           /* s_x */
    float inv_s_ln1;
    float alpha_1;                /* s_ln1 * s_w1 */
    float inv_s_ffn1;
    float alpha_2;                /* s_ffn1 * s_w2 */
    float resid2_scale;           /* s_ln1 */
    float inv_s_out;
    const nm_tables* tables;
    int32_t gelu_idx, exp_idx, recip_idx, rsqrt_idx;
    int32_t flags;                /* NM_LAYER_* (0: the library chooses) */
} nm_layer_desc;

/* Steps 5+6 and 8+9 as one kernel each (the LayerNorm runs in the epilogue of the matrix product,
 * on workgroups that own whole rows; the fp32 tensor between them never reaches memory).  Needs
 * H = 768 or 1024 and aligned operands; where that does not hold, or taps of the fp32 tensors are
 * asked for, the two-kernel path runs.  Results are identical either way. */
enum { NM_LAYER_FOLD_LAYERNORM = 1, NM_LAYER_NO_FOLD_LAYERNORM = 2 };

/* Optional device buffers that receive the intermediate tensors (any may be NULL; a non-NULL
 * buffer is used as that tensor's storage, so it costs nothing extra). */
typedef struct {
    int8_t* qkv;     /* [B*S, 3H] */
    int32_t* scores; /* [B, heads, S, S] */
    int8_t* p;       /* [B, heads, S, S] */
    int8_t* ctx;     /* [B*S, H] */
    float* attn;     /* [B*S, H] */
    int8_t* ln1;     /* [B*S, H] */
    int8_t* ffn1;    /* [B*S, F] */
    float* ffn2;     /* [B*S, H] */
} nm_layer_taps;

/* Bytes of device workspace nm_encoder_layer needs for this shape (host computation only). */
int32_t nm_encoder_layer_workspace(const nm_layer_desc* desc, size_t* bytes);

/*
 * x: device int8 [B*S, H].  y_q: device int8 [B*S, H] or NULL.  y_f32: device fp32 [B*S, H] or
 * NULL (at least one required).  ws: device workspace of at least the queried size, 256-byte
 * aligned; its contents are scratch.  taps may be NULL.
 * Limits: those of the calls above; H % heads == 0.
 */
int32_t nm_encoder_layer(const nm_layer_desc* desc, const int8_t* x, int8_t* y_q, float* y_f32,
                         void* ws, size_t ws_bytes, const nm_layer_taps* taps, void* stream);

/*
 * nm_encoder_layer_noalloc: nm_encoder_layer for callers that cannot allocate device memory (code
 * under HIP graph capture, tight serving loops, harnesses that forbid allocation): the workspace is
 * a buffer of NM_NOALLOC_MAX_WORKSPACE bytes built into the library's device image (each GPU the
 * library runs on holds one until the process ends), so the caller passes inputs and outputs only.
 * Same results as nm_encoder_layer, no taps.  Calls nothing that allocates or frees.
 * Returns NM_ERR_WORKSPACE (message says how much is needed) when nm_encoder_layer_workspace of
 * the shape exceeds NM_NOALLOC_MAX_WORKSPACE: B32 S128 H768 F3072 fits, B16 S512 H768 does not.
 * Every call on a GPU uses that GPU's one buffer, whose contents are scratch and survive from call
 * to call (nothing in it needs to start at zero): two calls that overlap in time on the same GPU,
 * from different streams or threads, race.  Calls on one stream are ordered and safe.
 */
#define NM_NOALLOC_MAX_WORKSPACE (64u << 20)
int32_t nm_encoder_layer_noalloc(const nm_layer_desc* desc, const int8_t* x, int8_t* y_q, float* y_f32,
                                 void* stream);

/* ---------------------------------------------------------------------------------------------
 * nm_encoder_stack: n_layers encoder layers back to back on one stream (the paper's Section 4
 * models are stacks of identical layers: 12 for BERT-base, 24 for BERT-large).  Layer l reads the
 * int8 output of layer l-1, so descs[l].resid1_scale / alpha_qkv must be formed from layer l-1's
 * output scale (the caller's job, as for every other multiplier).  All layers share B, S and H;
 * F and the tables may differ per layer.
 * descs: HOST array of n_layers descriptors (read during the call only).  x, y_q, y_f32 as for
 * nm_encoder_layer (y_f32 is the last layer's fp32 output).  If only y_f32 is given and
 * n_layers > 1 the intermediate layers still produce int8.  The workspace holds two activation
 * buffers plus the largest per-layer workspace; query it first.  Nothing is allocated and the
 * host does not wait for the GPU.
 * --------------------------------------------------------------------------------------------- */
int32_t nm_encoder_stack_workspace(const nm_layer_desc* descs, int32_t n_layers, size_t* bytes);
int32_t nm_encoder_stack(const nm_layer_desc* descs, int32_t n_layers, const int8_t* x, int8_t* y_q,
                         float* y_f32, void* ws, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------------------------
 * nm_conv2d_pwl: int8 convolution in its matrix form (paper Section 3.1: a convolution becomes a
 * matrix product whose dimensions follow from the width, height and channel counts) with the
 * epilogue of nm_gemm_pwl:
 *   acc[b,ho,wo,n] = sum_{i,j,c} x[b, ho*stride - pad + i, wo*stride - pad + j, c] * w[n,i,j,c]
 *                    (exact int32; positions outside the image contribute nothing)
 *   v = fma((float)acc, alpha_n, bias_n);  v = fma((float)resid, resid_scale, v) if resid;
 *   v = PWL(v) if table_idx >= 0 (ReLU is the exact two-segment table);  outputs v and its int8 code.
 * Ho = (H + 2*pad - kh) / stride + 1, Wo likewise.
 * x: device int8 [B, H, W, Cin] (channels contiguous).  w: device int8 [Cout, kh, kw, Cin].
 * bias, alpha_vec: device fp32 [Cout] or NULL (alpha_vec NULL -> alpha; a folded batch
 * normalisation is a per-channel alpha_vec and bias).  resid: device int8 [B, Ho, Wo, Cout] or
 * NULL.  Outputs (device, any may be NULL, at least one required): out_q int8, out_f32, dbg_acc
 * int32, each [B, Ho, Wo, Cout].
 * Workspace: needed only when Cin is not a multiple of 64 (or x / w are not 16-byte aligned) and
 * the convolution is not 1x1 / stride 1 / no padding (a patch matrix, or for images of at most
 * four channels a few KB for the repacked filter); query nm_conv2d_workspace (0 otherwise; ws may
 * then be NULL).  256-byte aligned, contents are scratch.  Nothing is allocated, the host
 * does not wait.  Limits: kh*kw*Cin <= 65536, B*Ho*Wo < 2^31, B*Ho*Wo*Cout < 2^31.
 * --------------------------------------------------------------------------------------------- */
typedef struct {
    int32_t B, H, W, Cin, Cout, kh, kw, stride, pad;
    const int8_t* x;
    const int8_t* w;
    const float* bias;
    const float* alpha_vec;
    float alpha;
    const int8_t* resid;
    float resid_scale;
    const nm_tables* tables;
    int32_t table_idx; /* -1: no table */
    float out_inv_scale;
    int8_t* out_q;
    float* out_f32;
    int32_t* dbg_acc;
} nm_conv_desc;

int32_t nm_conv2d_workspace(const nm_conv_desc* desc, size_t* bytes);
int32_t nm_conv2d_pwl(const nm_conv_desc* desc, void* ws, size_t ws_bytes, void* stream);

/*
 * nm_maxpool_i8: k x k max pooling on int8 codes that share one scale (exact; the paper does not
 * discuss pooling).  Positions outside the image never take part.  x: device int8 [B, H, W, C];
 * y: device int8 [B, Ho, Wo, C] with Ho = (H + 2*pad - k) / stride + 1.  Requires pad < k.
 */
int32_t nm_maxpool_i8(const int8_t* x, int32_t B, int32_t H, int32_t W, int32_t C, int32_t k,
                      int32_t stride, int32_t pad, int8_t* y, void* stream);

/*
 * nm_avgpool_i8: global average pooling as the linear operation it is (Section 3.1):
 * acc[b,c] = sum over the HW positions (exact int32), v = (float)acc * alpha with alpha =
 * s_x / HW formed by the caller, out_f32 = v, out_q = its int8 code.  x: device int8 [B, HW, C].
 */
int32_t nm_avgpool_i8(const int8_t* x, int32_t B, int32_t HW, int32_t C, float alpha, float out_inv_scale,
                      int8_t* out_q, float* out_f32, void* stream);

/* ---------------------------------------------------------------------------------------------
 * nm_cnn_run: a list of convolution / pooling / matrix-product steps queued back to back on one
 * stream (a whole residual CNN in one call; the steps are the entry points above, so results are
 * identical to calling them one by one).  ops: HOST array, read during the call only; every tensor
 * pointer inside is a device pointer owned by the caller, who also wires each step's input to an
 * earlier step's output.  ws: one workspace shared by all steps (query nm_cnn_workspace: the
 * largest any step needs).  Stops at the first failing step and returns its status.
 * --------------------------------------------------------------------------------------------- */
enum { NM_OP_CONV = 0, NM_OP_MAXPOOL = 1, NM_OP_AVGPOOL = 2, NM_OP_GEMM = 3 };

typedef struct {
    int32_t kind;                 /* NM_OP_* */
    nm_conv_desc conv;            /* NM_OP_CONV */
    nm_gemm_desc gemm;            /* NM_OP_GEMM */
    /* NM_OP_MAXPOOL: x [B,H,W,C] -> y, window k, stride, pad.  NM_OP_AVGPOOL: x [B,HW,C] (H = HW,
     * W unused), alpha, out_inv_scale -> y (int8) and / or y_f32. */
    const int8_t* x;
    int8_t* y;
    float* y_f32;
    int32_t B, H, W, C, k, stride, pad;
    float alpha, out_inv_scale;
} nm_cnn_op;

int32_t nm_cnn_workspace(const nm_cnn_op* ops, int32_t n_ops, size_t* bytes);
int32_t nm_cnn_run(const nm_cnn_op* ops, int32_t n_ops, void* ws, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------------------------
 * One step of a decoder over a paged key-value cache.
 *
 * The cache is a pool of num_pages pages of page_size slots (a power of two); a slot holds the key, and in the value cache the
 * value, of one token for all key heads.  Slot number = page * page_size + place in the page.  A request owns the pages that its row of
 * the block table names, in the order of its positions; position p of request b lies in slot
 * block_table[b][p / page_size] * page_size + p % page_size.  Element c of head h of a slot is at
 * page * page_stride + place * slot_stride + h * head_stride + c (strides in elements, alike for keys and values), so a page may be
 * laid out by tokens or by heads.  All of a step's numbers (lengths, slots, tables) are device memory, so that a step can
 * be captured once and replayed while they change.
 *
 * nm_qk_norm_rope and nm_paged_attention compute the functions themselves, not tables of them: a softmax that is split over the
 * cache's length and joined relies on exp(a + b) = exp(a) exp(b), which a piecewise-linear exp does not have.  nm_gemv_w4 takes tables.
 * Sums and statistics are binary32 (sums of up to 128 integer products exact int32); outputs are rounded once, to nearest even; int8 codes
 * as above.  The same call gives the same bits (no atomics); against the formulas results are right to rounding, not bit for bit.
 * Which kernels run depends on shapes and types alone, so every call can be captured; calls that overlap in time share nothing but
 * what the caller gives both.
 * --------------------------------------------------------------------------------------------- */

/*
 * nm_page_plan: block tables, slots and positions of a step from the requests' lengths.  Request b holds cached[b] tokens and adds
 * fresh[b] (0: idle).  With up(n) = ceil(n / page_size), it needs up(cached + fresh) - up(cached) new pages where fresh > 0; they come
 * from free_pages, from number *free_begin on, in the order of the requests, and are entered into its row behind the
 * up(cached) entries that are there.  Then, everything int32:
 *   lens[b] = cached[b] + fresh[b];  row_start[0 .. B] = prefix sums of fresh;  *free_end = *free_begin + pages taken;
 *   for token t, the i-th new one of request b:  requests[t] = b, positions[t] = cached[b] + i, slots[t] = its slot;
 *   rows behind the last token:  requests -1, positions 0, slots -1.
 * A token whose table or list entry is no page (outside [0, num_pages)) has slot -1.
 * status[0]: 0, or a sum of NM_PLAN_*; status[1]: new tokens, [2]: new pages needed, [3]: largest of cached + fresh (0 for B = 0); each at
 * most 2^31 - 1.  With any flag set nothing is assigned: the table is left as it is, slots and requests are -1, positions and
 * row_start 0, lens = cached, *free_end = *free_begin.  (The calls below leave rows without a slot out.)
 * cached, fresh: device [B].  free_pages: device [n_free].  block_table: device [B] rows of max_pages entries, table_stride
 * apart.  slots, positions, requests: [max_tokens].  lens, row_start, positions, requests may be NULL.  No output may be an input
 * (one workgroup writes while another still reads): *free_end and lens need memory of their own.
 * Limits: B <= NM_PLAN_MAX_REQUESTS; num_pages * page_size and max_pages * page_size < 2^31; page_size <= 65536; max_tokens, n_free <= 2^30.
 */
#define NM_PLAN_MAX_REQUESTS 4096
enum { NM_PLAN_NO_PAGES = 1,      /* the free list is too short */
       NM_PLAN_TABLE_FULL = 2,    /* a request needs more than max_pages entries */
       NM_PLAN_NO_ROWS = 4,       /* more than max_tokens new tokens */
       NM_PLAN_BAD_LENGTH = 8 };  /* a negative length, or *free_begin negative */
typedef struct {
    int32_t B, page_size, num_pages, max_pages, n_free, max_tokens;
    const int32_t* cached;
    const int32_t* fresh;
    const int32_t* free_pages;
    const int32_t* free_begin;
    int32_t* free_end;
    int32_t* block_table;
    int64_t table_stride;
    int32_t* lens;
    int32_t* row_start;
    int32_t* slots;
    int32_t* positions;
    int32_t* requests;
    int32_t* status; /* [4] */
} nm_plan_desc;

int32_t nm_page_plan(const nm_plan_desc* desc, void* stream);

/*
 * nm_qk_norm_rope: what lies between a step's QKV projection and its attention, in one pass.  For each of T tokens, hq heads of
 * queries and hk of keys, d elements each:
 *   y = x / sqrt(mean(x^2) + eps) * gamma     with NM_QK_NORM (gamma NULL: 1), else y = x
 *   the first rot elements are turned by the angles a_i = position * inv_freq[i], i < rot / 2 (products exact to 2^-53):
 *   (y_p, y_q) -> (y_p cos a_i - y_q sin a_i, y_q cos a_i + y_p sin a_i),  p, q = i, i + rot / 2, or 2 i, 2 i + 1 with NM_ROPE_INTERLEAVED
 * Queries go to q_out; keys to k_out (may be NULL) and, with the values as they are, to their token's slot of the cache (k_cache and
 * v_cache both NULL: no cache, v is not read).  int8 caches hold codes: clamp(rint(value * inv_scale[head]), -127, 127).
 * A slot outside [0, num_pages * page_size) is not written.  Two tokens of one slot: every element is one of the two's.
 * q, k, v: device, a token's heads one behind the other, tokens q_stride, k_stride, v_stride elements apart (the thirds of a fused
 * projection's rows, for instance); in_dtype F32, BF16 or F16.  q_out, k_out likewise, out_dtype the same three; q_out may be q itself
 * (same type and stride), k_out k; no other output may be an input or another output.  cache_dtype F32, BF16, F16 or I8.  positions, slots: device int32 [T] (positions may be NULL for rot = 0,
 * slots without a cache).  Rows without a slot are computed into q_out and k_out like the others.  inv_freq: device fp32 [rot / 2].  gammas: device fp32 [d].  k_inv_scale, v_inv_scale: device fp32 [hk], for int8.
 * Limits: T <= 2^23; 1 <= d <= 256; rot even, 0 <= rot <= d; hq, hk >= 1, hq + 2 hk <= 65535; strides cover a token's heads.  Where the rows and the cache are
 * 16-byte aligned, d is a multiple of 8 and rot of 8 (or 0), whole groups of elements move at once.
 */
enum { NM_QK_NORM = 1, NM_ROPE_INTERLEAVED = 2 };
typedef struct {
    int32_t T, hq, hk, d, rot, flags;
    int32_t in_dtype, out_dtype, cache_dtype;
    int32_t num_pages, page_size;
    const void* q; const void* k; const void* v;
    int64_t q_stride, k_stride, v_stride;
    const float* q_gamma;
    const float* k_gamma;
    float eps;
    const int32_t* positions;
    const float* inv_freq;
    void* q_out;
    int64_t q_out_stride;
    void* k_out;
    int64_t k_out_stride;
    void* k_cache;
    void* v_cache;
    int64_t page_stride, slot_stride, head_stride;
    const int32_t* slots;
    const float* k_inv_scale;
    const float* v_inv_scale;
} nm_qk_desc;

int32_t nm_qk_norm_rope(const nm_qk_desc* desc, void* stream);

/*
 * nm_paged_attention: attention of one new token of every request over the request's cache.  With n = lens[b], the query heads
 * h of a group sharing key head g = h / (hq / hk), and the positions j in [max(0, n - window), n) (window 0: [0, n)):
 *   s_j = scale * q[b,h] . k_j        k_j, v_j: key and value of position j for head g, int8 codes times k_scale[g], v_scale[g]
 *   out[b,h] = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),  m = max_j s_j;   lse[b,h] = m + log sum_j exp(s_j - m)
 * No position (n <= 0): out 0, lse -inf.  A length beyond max_pages * page_size counts as that; a position whose table entry
 * is no page (outside [0, num_pages)) takes no part.  Slots behind a request's length are never read: what they hold does not matter.
 * q: device [B, hq, d], requests q_stride elements apart, q_dtype F32, BF16 or F16.  Cache: as above, cache_dtype BF16, F16 or I8
 * (then k_scale, v_scale: device fp32 [hk]).  block_table: device int32, rows of max_pages entries table_stride apart.  lens:
 * device int32 [B].  out: device [B, hq, d], requests out_stride apart, out_dtype F32, BF16, F16 or I8 (codes with
 * out_inv_scale: what nm_gemm_pwl reads); out may be q itself (same type and stride), and is no other input.  lse: device fp32 [B, hq] or NULL; neither an
 * input nor out.
 * q is split into as many terms of the matrix instructions' type as hold it, the weights into two (fp32 results: three), so nothing
 * but the outputs is rounded to fewer than 16 bits.
 * Workspace: query nm_paged_attention_workspace (it looks at the description's sizes, strides and types, never at device memory; 0: none); 256-byte
 * aligned, contents are scratch, calls that overlap in time need one each.  Lengths may be as ragged, and the table as much wider
 * than they are, as it happens: the work is shared by the lengths as they are when the call runs.
 * Limits: hq % hk == 0; d a multiple of 16 up to 256; cache addresses and strides multiples of 16 bytes; page_size a power of
 * two up to 65536; num_pages * page_size < 2^31; max_pages * page_size < 2^30; each cache at most 32 GiB; B * hq < 2^23.
 */
typedef struct {
    int32_t B, hq, hk, d;
    int32_t q_dtype, cache_dtype, out_dtype;
    int32_t page_size, num_pages, max_pages;
    const void* q;
    int64_t q_stride;
    const void* k_cache;
    const void* v_cache;
    int64_t page_stride, slot_stride, head_stride;
    const float* k_scale;
    const float* v_scale;
    const int32_t* block_table;
    int64_t table_stride;
    const int32_t* lens;
    float scale;
    int32_t window;
    void* out;
    int64_t out_stride;
    float out_inv_scale;
    float* lse;
} nm_paged_desc;

int32_t nm_paged_attention_workspace(const nm_paged_desc* desc, size_t* bytes);
int32_t nm_paged_attention(const nm_paged_desc* desc, void* ws, size_t ws_bytes, void* stream);

/*
 * nm_gemv_w4: product of a few rows with 4-bit weights, the projections of a step.
 *   acc[m,n] = sum over groups g of scales[n,g] * sum_{k in g} x[m,k] * w[n,k]      (int8 x: of a group, or of 128 of its products at a time, exact in int32)
 *   v = fma(acc, alpha, bias_n);  v = PWL_table(v) if table_idx >= 0;  out[m,n] = v, or its int8 code with out_inv_scale
 * x: device [M, K], rows x_stride elements apart, x_dtype I8, BF16 or F16.  W: device [N, K / 2], contiguous: byte i of a row holds
 * w[n, 2 i] in its low and w[n, 2 i + 1] in its high four bits, two's complement (-8 .. 7).  scales: device [N, K / group], contiguous,
 * scale_dtype F32, BF16 or F16.  bias: device fp32 [N] or NULL.  out: device [M, N], rows out_stride apart, out_dtype F32, BF16, F16
 * or I8; out is none of the inputs.  Any M: rows are taken up to 48 at a time, and the weights read again for each (many rows are better off with nm_gemm_pwl
 * and int8 weights).
 * bf16 and fp16 rows meet the weights themselves, in exact products: a value whose weight is zero leaves no error, an infinity follows the
 * formula (times a weight of zero: NaN), and neither it nor a NaN reaches another row.
 * Limits: group 32, 64 or a multiple of 128; K a multiple of group, at most 65536; x and W 16-byte aligned, x_stride a multiple of 16
 * bytes; M <= 2^20, N < 2^26, (N / 16) (M / 32) < 2^23.
 */
typedef struct {
    int32_t M, N, K, group;
    int32_t x_dtype, scale_dtype, out_dtype;
    const void* x;
    int64_t x_stride;
    const uint8_t* W;
    const void* scales;
    float alpha;
    const float* bias;
    const nm_tables* tables;
    int32_t table_idx; /* -1 = no nonlinearity */
    void* out;
    int64_t out_stride;
    float out_inv_scale;
} nm_w4_desc;

int32_t nm_gemv_w4(const nm_w4_desc* desc, void* stream);

/* ---------------------------------------------------------------------------------------------
 * Several hypotheses per request over the paged cache: a row of the batch is a hypothesis, and the rows of a request share the pages of
 * what they have in common.  One step: nm_page_plan (one new token per row), the model with nm_qk_norm_rope and nm_shared_attention,
 * nm_beam_select over its logits, nm_page_fork, and nm_page_copy of the pages that it names, before pages are taken again.  As above, a step's
 * numbers are device memory, nothing is allocated, the host does not wait, every call can be captured, and the same call gives the same bits.
 * Workspaces: 256-byte aligned, contents are scratch, calls that overlap in time need one each.
 * --------------------------------------------------------------------------------------------- */

/*
 * nm_beam_select: the K best continuations of each of R requests with W hypotheses.  Row r W + w of the logits belongs to
 * hypothesis w of request r, whose log-probability so far is scores[r,w]:
 *   t(w, v) = scores[r,w] + x[w,v] - log sum_u exp(x[w,u])    for the tokens v of every hypothesis with done[r,w] = 0
 *   t(w, end_token) = scores[r,w]                            the only candidate of one with done[r,w] != 0
 * The K candidates of largest weight[r,w] * t go out, best first (weight NULL: 1); equal ones by w, then by logit, then by v, the lowest first
 * (the largest logit).  For the k-th:  parents[r,k] = r W + w;  tokens[r,k] = v;  scores_out[r,k] = t;
 * done_out[r,k] = done[r,w] != 0 or v == end_token.  Fewer than K candidates: parents and tokens -1, scores_out -inf, done_out 0.
 * No candidates: tokens whose logit is -inf or NaN (masked), and hypotheses whose score or weight is not finite, or whose weight is not above 0.
 * A logit of +inf counts as the largest binary32 number.  Logits are compared as they are; t and weight * t are formed in 64 bits from a sum of exponentials
 * in 32 (partial sums of up to 16 terms, joined in 64), whose logarithm is right to 2^-18, so that of two hypotheses' candidates whose weight * t are closer than 2^-17 times the larger
 * weight either may come first, but always the same.
 * history (NULL: none): row r W + w holds the history_lens[r W + w] tokens of that hypothesis, in rows of max_history.  Row r K + k of history_out receives
 * its parent's tokens and, unless the parent was done or the row is full, the new one; history_lens_out how many these are (no parent: 0).  What is behind
 * them is left as it was.  Lengths outside [0, max_history] count as the nearest.
 * logits: device [R W, V], rows logits_stride elements apart, logits_dtype F32, BF16 or F16.  scores, weight: device fp32 [R, W]; done: device int32 [R, W] or
 * NULL.  parents, tokens, done_out (or NULL): device int32 [R, K]; scores_out: device fp32 [R, K].  history, history_out: device int32, rows
 * history_stride and history_out_stride apart; history_lens, history_lens_out: device int32 [R W], [R K].  No output may be an input or another output.
 * Limits: 1 <= W, K <= NM_BEAM_MAX; R W <= 2^20; R K <= 2^23; 1 <= V <= 2^26; 1 <= max_history <= 2^30.  -1 <= end_token < V (-1: none; then done is NULL).
 */
#define NM_BEAM_MAX 64
typedef struct {
    int32_t R, W, K, V;
    int32_t logits_dtype, end_token, max_history;
    const void* logits;
    int64_t logits_stride;
    const float* scores;
    const float* weight;
    const int32_t* done;
    int32_t* parents;
    int32_t* tokens;
    float* scores_out;
    int32_t* done_out;
    const int32_t* history;
    int64_t history_stride;
    const int32_t* history_lens;
    int32_t* history_out;
    int64_t history_out_stride;
    int32_t* history_lens_out;
} nm_beam_desc;

int32_t nm_beam_select_workspace(const nm_beam_desc* desc, size_t* bytes);
int32_t nm_beam_select(const nm_beam_desc* desc, void* ws, size_t ws_bytes, void* stream);

/*
 * nm_page_fork: the block tables of a new batch whose row b goes on from row parents[b] of the old one.  A parent outside [0, B_in)
 * leaves row b empty; a row may have several children (they share its pages), one (it moves) or none (what only it held becomes free), and B_out
 * may differ from B_in (a batch is compacted, or grows).  Old row r holds lens[r] tokens in its first up(lens) = ceil(lens / page_size) entries.
 * For row b of parent p, and n = lens[p]:  lens_out[b] = n;  the first up(n) entries of its row of table_out are p's, but for the last
 * page where n is no multiple of page_size: the next token would be written into it.  It stays p's page for the lowest-numbered row with
 * that parent, if no other old row with children refers to the page and keep (NULL: nobody) is 0 for it; every other row gets a page of its own: the next of
 * free_pages, from number *free_begin on, in the order of the rows.  copy_src[b], copy_dst[b] and copy_slots[b] then say which page's first
 * slots are to be copied where (nm_page_copy), and are -1, -1, 0 for the other rows.  Entries behind up(n) are left as they were.
 * Pages that old rows refer to and no new row does, and that keep does not hold (keep[page] != 0: a page of a prefix cache, or of another batch), are
 * freed: with `taken` pages taken and `freed` freed, *free_end = *free_begin + taken - freed, and free_out holds from there the freed pages, ascending, and then
 * the rest of free_pages as it was.  What lies in front of *free_end is left as it was.  free_out may be free_pages.
 * A copied page that is freed keeps its contents until pages are taken again: copy before that.
 * Entries that are no pages (outside [0, num_pages)) are handed on, and neither copied nor freed.
 * status[0]: 0, or a sum of NM_FORK_*; [1]: pages wanted, [2]: pages freed, [3]: rows with a parent.  With any flag set nothing is assigned:
 * table_out is left as it is, lens_out is 0, there are no copies, free_out holds the rest of free_pages, and *free_end = *free_begin.
 * (With NM_FORK_BAD_LENGTH the other numbers and flags count only the rows whose length is good.)
 * lens: device int32 [B_in].  parents: [B_out].  block_table, table_out: int32, rows of max_pages entries, table_stride and table_out_stride
 * apart.  keep: int32 [num_pages] or NULL.  free_pages, free_out: [n_free].  lens_out, copy_src, copy_dst, copy_slots: [B_out].  Apart from free_out no output may be an
 * input, and none another output.
 * Limits: B_in, B_out <= NM_PLAN_MAX_REQUESTS; page_size a power of two up to 65536; num_pages * page_size and max_pages * page_size < 2^31; num_pages, max_pages,
 * n_free <= 2^30.
 */
enum { NM_FORK_NO_PAGES = 1,      /* the free list is too short */
       NM_FORK_BAD_LENGTH = 8,    /* a length that is negative or longer than max_pages, or *free_begin outside [0, n_free] */
       NM_FORK_LIST_FULL = 16 };  /* the list has no room in front of *free_begin for the pages that become free */
typedef struct {
    int32_t B_in, B_out, page_size, num_pages, max_pages, n_free;
    const int32_t* block_table;
    int64_t table_stride;
    const int32_t* lens;
    const int32_t* parents;
    const int32_t* keep;
    const int32_t* free_pages;
    const int32_t* free_begin;
    int32_t* table_out;
    int64_t table_out_stride;
    int32_t* lens_out;
    int32_t* free_out;
    int32_t* free_end;
    int32_t* copy_src;
    int32_t* copy_dst;
    int32_t* copy_slots;
    int32_t* status; /* [4] */
} nm_fork_desc;

int32_t nm_page_fork_workspace(const nm_fork_desc* desc, size_t* bytes);
int32_t nm_page_fork(const nm_fork_desc* desc, void* ws, size_t ws_bytes, void* stream);

/*
 * nm_page_copy: copies pages inside each of n_caches caches of one layout (a model's key and value caches of every layer): for i < n, the first
 * slots[i] slots (NULL: page_size; more counts as page_size, fewer than 1 as none) of page src[i] to page dst[i].  A copy whose src or dst is no page (outside [0, num_pages)), or
 * that are one page, is left out.  No page may be the destination of two copies, or the source of one and the destination of another: what those
 * hold is not said then.
 * caches: HOST array of n_caches device pointers, read during the call.  dtype: F32, BF16, F16 or I8; elements are moved as they are.  src, dst,
 * slots: device int32 [n].  Strides as above, in elements.  Where addresses, strides and rows are multiples of 16 bytes, whole groups of 16 bytes move at once (else as wide ones as they allow).
 * Limits: n <= 2^20; n_caches <= NM_COPY_MAX_CACHES; page_size a power of two up to 65536; hk, d >= 1; num_pages * page_size, and
 * page_size * hk * d, < 2^31; each of the n pages in pieces of 1024 such groups, fewer than 2^24 pieces in all.
 */
#define NM_COPY_MAX_CACHES 256
typedef struct {
    int32_t n, n_caches, hk, d, dtype;
    int32_t num_pages, page_size;
    void* const* caches;
    int64_t page_stride, slot_stride, head_stride;
    const int32_t* src;
    const int32_t* dst;
    const int32_t* slots;
} nm_copy_desc;

int32_t nm_page_copy(const nm_copy_desc* desc, void* stream);

/*
 * nm_shared_attention: nm_paged_attention where groups of rows share a prefix, which is read once for all of a group's rows.  Group g is the rows
 * group_start[g] .. group_start[g + 1] - 1, and the keys and values of the first shared[g] positions are the same for all of its rows (as nm_page_fork leaves
 * them; a shared end inside a page is possible).  Which of the rows' entries they are read through is not said.
 * A row shorter than its group's shared[g] takes no part in that and is computed by itself, as is a row of no group.  shared[g] < 1: nothing is shared.
 * If group_start does not ascend, or leaves [0, B], no row is in a group.
 * desc->p: as for nm_paged_attention, its outputs and limits likewise, but window is 0 (rows of a window share little: nm_paged_attention).  group_start: device
 * int32 [G + 1]; shared: device int32 [G].
 * Limits besides: B <= NM_PLAN_MAX_REQUESTS, G <= NM_PLAN_MAX_REQUESTS.
 */
typedef struct {
    nm_paged_desc p;
    int32_t G;
    const int32_t* group_start;
    const int32_t* shared;
} nm_shared_desc;

int32_t nm_shared_attention_workspace(const nm_shared_desc* desc, size_t* bytes);
int32_t nm_shared_attention(const nm_shared_desc* desc, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* NM_H */
