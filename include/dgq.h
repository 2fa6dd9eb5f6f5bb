/*
 * dgq.h - C ABI of the B200 (sm_100a) hot path of DGQ, distribution-aware group
 * quantization for text-to-image diffusion models.
 *
 * Equations of the paper are unnumbered; they are numbered here in order of
 * appearance: Eq. 1 linear quantizer, Eq. 2 log quantizer (Sec. 3.1); Eq. 3
 * softmax attention score (Sec. 3.2); Eq. 4 range-variability metric D_d,
 * Eq. 5 d* = argmax D_d, Eq. 6 per-group scale and zero-point, Eq. 7
 * per-timestep parameter sets, Eq. 8 log-quantized cross-attention codes,
 * Eq. 9 split product A_hat V_hat (Sec. 3.3).
 *
 * Conventions
 *  - "dev" pointers are CUDA device memory owned by the caller; "host" pointers
 *    are ordinary host memory owned by the caller.  The library never frees or
 *    keeps a caller's pointer beyond the call.
 *  - `stream` is a cudaStream_t passed as void* (NULL = the default stream).
 *  - Every function returns a dgq_status.  Nothing throws, aborts or prints.
 *    There is no CPU fallback: unsupported shapes or alignments are errors.
 *  - dgq_quantize_act, dgq_linear and dgq_cross_attn_logq only enqueue work on
 *    `stream`; they allocate nothing and do not synchronise.  The calibration
 *    and weight-preparation calls allocate library-owned objects and
 *    synchronise with the host.
 *  - The kernels these three calls enqueue are launched so that the next kernel
 *    on the stream may be scheduled while the current one finishes; each waits
 *    for everything enqueued before it on the stream before it reads or writes
 *    memory, so stream order is kept as with ordinary launches, also inside a
 *    captured CUDA graph.  Setting DGQ_PDL=0 in the environment before the
 *    first call falls back to ordinary launches.
 *  - Device-side waits are bounded.  A kernel that gives up on a wait records
 *    DGQ_ERR_TIMEOUT in a device status word read by dgq_device_status().
 */
#ifndef DGQ_H_
#define DGQ_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int dgq_status;
enum {
  DGQ_OK = 0,
  DGQ_ERR_INVALID_ARG = 1,   /* NULL pointer, non-positive size, unknown enum, timestep out of range */
  DGQ_ERR_ALIGNMENT = 2,     /* pointer not 16-byte aligned or leading dimension not a multiple of 8 elements */
  DGQ_ERR_UNSUPPORTED = 3,   /* valid request outside what the kernels implement (stated per call) */
  DGQ_ERR_WORKSPACE = 4,     /* workspace missing or too small */
  DGQ_ERR_CUDA = 5,          /* a CUDA runtime / driver call failed */
  DGQ_ERR_TIMEOUT = 6,       /* a bounded device-side wait gave up (see dgq_device_status) */
  DGQ_ERR_NOT_CALIBRATED = 7 /* the table row of the requested timestep was never filled */
};

/* dim_select / dgq_groups_info dim */
enum { DGQ_DIM_AUTO = 0, DGQ_DIM_CHANNEL = 1, DGQ_DIM_PIXEL = 2, DGQ_DIM_BOTH = 3 };
/* outlier_mode */
enum { DGQ_OUTLIER_KMEANS = 0, DGQ_OUTLIER_EXPLICIT = 1 };
/* quantizer parameter source */
enum { DGQ_MODE_STATIC = 0, DGQ_MODE_DYNAMIC_TOKEN = 1 };
/* code layout written by dgq_quantize_act and read by dgq_linear */
enum { DGQ_CODES_U8 = 0, DGQ_CODES_S8_CENTRED = 1 };
/* scope of the maximum in Eq. 8 */
enum { DGQ_SCALE_PER_PROMPT = 0, DGQ_SCALE_PER_PROMPT_HEAD = 1, DGQ_SCALE_PER_CALL = 2 };

#define DGQ_MAX_GROUPS 32    /* groups along either dimension */
#define DGQ_K_ATOM 32        /* every channel group is padded to a multiple of this many codes */

/* Library-owned, opaque.  Created by the call that returns them, freed by *_destroy. */
typedef struct dgq_groups dgq_groups; /* grouping of one layer + per-timestep (s, 1/s, Z) tables */
typedef struct dgq_weight dgq_weight; /* low-bit weight of one layer in the kernel's layout */

typedef struct {
  int act_bits;        /* b of Eq. 1 / Eq. 6: 2..8 */
  int n_groups;        /* K of the K-means grouping, 1..DGQ_MAX_GROUPS-1 */
  int dim_select;      /* DGQ_DIM_AUTO (Eq. 5) or a forced dimension; DGQ_DIM_BOTH groups both */
  int outlier_mode;    /* DGQ_OUTLIER_KMEANS (the paper) or DGQ_OUTLIER_EXPLICIT (one extra group) */
  float outlier_tau;   /* EXPLICIT: a vector is an outlier if its range width > tau * median width */
  int n_timesteps;     /* T of Eq. 7: number of table rows */
  int rows_per_sample; /* P: pixels (tokens) per sample; row i is pixel position i mod P */
} dgq_calib_config;

typedef struct { int n, h, w, c; } dgq_conv_desc; /* NHWC input of a 3x3, stride 1, zero-pad 1 conv */

/* ---------------------------------------------------------------- calibration (Sec. 3.3, Eq. 4-7)
 * X_cal: dev fp16 [n_rows, C] row-major with leading dimension `ld` elements;
 * n_rows a multiple of rows_per_sample.
 * *inout == NULL: computes per-channel and per-pixel extrema (Eq. 4), picks d*
 *   (Eq. 5) unless forced, groups the vectors along it by K-means on their
 *   (min, max) range, fixes the grouping and the padded code layout for the
 *   layer, fills table row `timestep` from the cells' ranges (Eq. 6) and returns
 *   a new object in *inout.
 * *inout != NULL: keeps the grouping and (re)fills table row `timestep` (Eq. 7).
 * Synchronous with the host (the grouping runs on the host).
 * Errors: INVALID_ARG, ALIGNMENT, UNSUPPORTED (C > 8192), CUDA. */
dgq_status dgq_calibrate_groups(const dgq_calib_config* cfg, const void* X_cal, int64_t n_rows, int C,
                                int64_t ld, int timestep, dgq_groups** inout, void* stream);

/* Builds the same object from host arrays (for tables calibrated elsewhere).
 * col_group[C] in [0,G), row_group[P] in [0,R); scale[T*R*G] (fp32, > 0) and
 * zp[T*R*G]; every row counts as filled.  1/s is recomputed in fp32. */
dgq_status dgq_groups_from_host(int C, int P, int act_bits, int G, int R, int T, const int32_t* col_group,
                                const int32_t* row_group, const float* scale, const int32_t* zp,
                                dgq_groups** out);
dgq_status dgq_groups_destroy(dgq_groups* g);
/* Any out pointer may be NULL.  K_pad = length of one padded code row. */
dgq_status dgq_groups_info(const dgq_groups* g, int* C, int* P, int* K_pad, int* G, int* R, int* T,
                           int* dim, int* act_bits, double* D_channel, double* D_pixel);
/* Copies to host arrays (any may be NULL): perm[K_pad] = channel stored at each
 * padded position, -1 for padding; col_group[C]; group_off[G+1] = first padded
 * position of each group; row_group[P]; scale, zp [T*R*G]. */
dgq_status dgq_groups_export(const dgq_groups* g, int32_t* perm, int32_t* col_group, int32_t* group_off,
                             int32_t* row_group, float* scale, int32_t* zp);

/* ---------------------------------------------------------------- activation quantizer (Eq. 1 with Eq. 6)
 * X: dev fp16 [M, C], leading dimension `ld` (for a conv input: NHWC flattened
 * to [n*h*w, C]).  Xq: dev bytes [M, K_pad], channels permuted group-contiguous,
 * each group padded to a multiple of DGQ_K_ATOM.
 *   q = clamp(rint(x * inv_s) + Z, 0, 2^b - 1) in fp32, with (inv_s, Z) of the
 *   cell (pixel group of row i mod P, channel group of the column).
 * DGQ_MODE_STATIC: parameters from table row `timestep`.
 * DGQ_MODE_DYNAMIC_TOKEN: Eq. 6 applied to each token's members of each channel
 *   group; the parameters are written to dyn_scale, dyn_zp (dev [M, G]) for
 *   dgq_linear.  Inputs must be finite.
 * DGQ_CODES_U8 stores q (padding = Z); DGQ_CODES_S8_CENTRED stores q - Z as a
 *   signed byte (padding = 0) and needs L - 127 <= Z <= 128 for every cell,
 *   else UNSUPPORTED (static mode only).
 * Errors: INVALID_ARG, ALIGNMENT, NOT_CALIBRATED, UNSUPPORTED, CUDA. */
dgq_status dgq_quantize_act(const dgq_groups* g, int timestep, int mode, int layout, const void* X, int64_t M,
                            int64_t ld, void* Xq, float* dyn_scale, int32_t* dyn_zp, void* stream);

/* ---------------------------------------------------------------- weights (offline)
 * Per-out-channel symmetric round-to-nearest codes (stands in for the paper's
 * BRECQ / AdaRound weights, Sec. 4.1), permuted and padded to the layer's code
 * layout, int4 packed two per byte, with the per-group column sums the
 * de-quantizer needs.  W: dev fp16 [N, K] (K = C), or [N, 3, 3, C] when conv is
 * non-NULL.  w_bits 8 or 4.  Synchronous with the host. */
dgq_status dgq_weight_prepare(const dgq_groups* g, const void* W, int N, int K, int w_bits,
                              const dgq_conv_desc* conv, dgq_weight** out, void* stream);
/* The same from codes quantized elsewhere: wq host int8 [N, K] (or [N,3,3,C]),
 * sw host fp32 [N]. */
dgq_status dgq_weight_from_codes(const dgq_groups* g, const int8_t* wq, const float* sw, int N, int K,
                                 int w_bits, const dgq_conv_desc* conv, dgq_weight** out);
dgq_status dgq_weight_destroy(dgq_weight* w);
/* Host copies of the codes in original channel order (int8 [N, K]) and scales.  Reads the weight's own device
 * whichever is current, waits for none of the caller's streams and may be called while the calling thread captures one. */
dgq_status dgq_weight_export(const dgq_weight* w, int8_t* wq, float* sw);

/* ---------------------------------------------------------------- group-quantized layer
 * Y[t, o] = bias[o] + sw[o] * sum_g s[t, g] * ( acc_g[t, o] - Z[t, g] * wsum_g[o] ),
 * acc_g the int32 product of the codes of channel group g with the weight codes
 * (Eq. 1's de-quantizer applied per group; the tensor-core accumulator is
 * switched at every group boundary).  Xq as written by dgq_quantize_act in
 * `layout`.  STATIC: (s, Z) of table row `timestep`, cell of (row mod P, g).
 * DYNAMIC_TOKEN: dyn_scale, dyn_zp dev [M, G].  bias dev fp16 [N] or NULL.
 * Y dev fp16 [M, N] with leading dimension ldy.  conv != NULL: 3x3 stride-1
 * zero-padded convolution of the NHWC code tensor as an implicit GEMM; needs
 * the S8_CENTRED layout, STATIC mode and channel-only grouping (R = 1).
 * workspace: dev, 256-byte aligned, at least dgq_linear_workspace_bytes(); only
 * 4-bit weights need one (a kernel in front of the GEMM expands them to bytes
 * there, once per call instead of once per row tile; the bytes stay in L2).
 * Contents undefined on entry and exit; calls that may overlap on the GPU need
 * separate workspaces unless they use the same weight.  NULL / 0 for 8-bit
 * weights.  NULL with 4-bit weights is allowed: the GEMM then expands the
 * weights itself, stage by stage and once per row tile, as it also does with a
 * workspace where that is faster (small problems); a non-NULL workspace that is
 * too small is an error.
 * Errors: INVALID_ARG, ALIGNMENT, NOT_CALIBRATED, WORKSPACE, UNSUPPORTED (K_pad *
 * 255 * 127 would overflow int32; more column blocks of 128 outputs, 160 where that
 * divides N, than the GPU has SMs; conv shape outside the supported tiling), CUDA. */
dgq_status dgq_linear(const dgq_groups* g, const dgq_weight* w, int timestep, int mode, int layout,
                      const void* Xq, const float* dyn_scale, const int32_t* dyn_zp, const void* bias,
                      void* Y, int64_t M, int64_t ldy, const dgq_conv_desc* conv, void* workspace,
                      size_t workspace_bytes, void* stream);
/* Bytes of workspace dgq_linear needs for this weight and M rows (0 for 8-bit weights). */
dgq_status dgq_linear_workspace_bytes(const dgq_groups* g, const dgq_weight* w, int64_t M, size_t* bytes);

/* ---------------------------------------------------------------- cross-attention (Eq. 3, 8, 9)
 * Q dev fp16 [B, nq, H, d]; K, V dev fp16 [B, nk, H, d]; O dev fp16 [B, nq, H, d].
 * A = softmax(Q K^T / sqrt(d)) in fp32; s = max of A over the columns j >= 1
 * within `scale_gran`; codes = clamp(rint(-log2(A / s)), 0, 2^bits - 1) for
 * j >= 1; O = A[:, 0] V[0] + s * sum_{j>=1} 2^-code V[j].  Column 0 (<start>)
 * stays in fp32.  fixed_scale (dev, [B], [B*H] or [1] by granularity) replaces
 * the dynamic maximum when non-NULL.  scale_out (same shape) and codes_out
 * (dev u8 [B, H, nq, nk-1]) are optional outputs.
 * workspace: dev, at least dgq_cross_attn_workspace_bytes(); contents undefined
 * on entry.  d a multiple of 8, d <= 160, 2 <= nk <= 128.
 * One kernel: with a dynamic scale its thread blocks exchange their maxima
 * through the workspace and meet at a grid barrier, so it is launched
 * cooperatively (and, inside a stream capture, becomes a cooperative kernel
 * node); grids larger than one resident wave run as two ordinary kernels.
 * Errors: INVALID_ARG (nk < 2), ALIGNMENT, UNSUPPORTED, WORKSPACE, CUDA. */
dgq_status dgq_cross_attn_logq(const void* Q, const void* K, const void* V, int B, int H, int nq, int nk,
                               int d, int score_bits, int scale_gran, const float* fixed_scale, void* O,
                               float* scale_out, uint8_t* codes_out, void* workspace,
                               size_t workspace_bytes, void* stream);

/* The same attention with a quantized value operand V_hat (Eq. 9 writes the product as A_hat V_hat
 * without naming V's quantizer).  Reading taken here: Eq. 1 with the range of Eq. 6 over one
 * head's [nk, d] slab of one prompt at `v_bits` (2..8) bits, code decided in fp32,
 * V_hat = s (q - Z); rows j >= 1 enter the product as fp16, row 0 (<start>) in fp32.  Everything
 * else, workspace included, as for dgq_cross_attn_logq.  Errors: as there, INVALID_ARG also for
 * v_bits outside 2..8. */
dgq_status dgq_cross_attn_logq_qv(const void* Q, const void* K, const void* V, int B, int H, int nq, int nk,
                                  int d, int score_bits, int scale_gran, const float* fixed_scale, int v_bits,
                                  void* O, float* scale_out, uint8_t* codes_out, void* workspace,
                                  size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------- self-attention (Eq. 2, Eq. 3; Sec. 3.3
 * applies the log quantizer "to both self and cross-attentions")
 * Q dev fp16 [B, nq, H, d]; K, V dev fp16 [B, nk, H, d]; O dev fp16 [B, nq, H, d]; any nk >= 1.
 * A = softmax(Q K^T / sqrt(d)) in fp32; codes = clamp(rint(-log2(A / s)), 0, 2^bits - 1) over ALL keys
 * (there is no <start> column here); O = s * sum_j 2^-code_j V[j].  s is the largest score of each query
 * row, or fixed_scale[b] (dev [B]) when non-NULL; the paper states the dynamic scale for cross-attention
 * only, the row maximum is this library's reading.  codes_out (dev u8 [B, H, nq, nk]) is optional.
 * No workspace: the keys are walked twice by the same thread block.  d in {40, 64, 80, 128, 160}.
 * Errors: INVALID_ARG, ALIGNMENT, UNSUPPORTED, CUDA. */
dgq_status dgq_self_attn_logq(const void* Q, const void* K, const void* V, int B, int H, int nq, int nk, int d,
                              int score_bits, const float* fixed_scale, void* O, uint8_t* codes_out, void* stream);
dgq_status dgq_cross_attn_workspace_bytes(int B, int H, int nq, int nk, int d, size_t* bytes);

/* ---------------------------------------------------------------- attention over an encoder's states and over an 8-bit cache
 * (The paper leaves text keys and values as they come from the encoder: one length, 16 bits.  The calls of this section
 * are this library's own: prompts of different lengths, and their keys and values kept in 8 bits over all steps.)
 * Like the hot-path calls above, all of them only enqueue work on `stream`: they allocate nothing, need no workspace and
 * do not synchronise.  Work goes to the current device, where all memory has to be. */

/* element type of the 16-bit tensors */
enum { DGQ_F16 = 0, DGQ_BF16 = 1 };

/* A 16-bit tensor [batch, tokens, heads, d], dev.  The d values of a row lie next to each other; the strides count
 * elements and may be those of a view (a slice of a fused projection, [batch, heads, tokens, d] storage).  `ptr` is 16-byte
 * aligned and strides are multiples of 8, else DGQ_ERR_ALIGNMENT; the stride of a dimension of size 1 is ignored.  Of
 * tensors that are read, batch and head strides may be 0 (one prompt's states for a whole batch); no stride is negative. */
typedef struct {
  void* ptr;
  int64_t batch, token, head;
} dgq_rows;

/* O[b, i, h] = sum_j softmax_j(scale Q[b, i, h] . K[b, j, h / (Hq / Hkv)]) V[b, j, h / (Hq / Hkv)] over the first
 * kv_lens[b] of the nk keys (dev int32 [B]; values outside 0..nk are taken as the nearer end; NULL: all nk), with scores and
 * softmax statistics in fp32 and weights rounded to the tensors' type for the product.  A request without keys gives zeros.
 * What K and V hold behind kv_lens[b] may be anything, NaN included.  Q, O [B, nq, Hq, d]; K, V [B, nk, Hkv, d]; Hq a
 * multiple of Hkv; d a multiple of 8 up to 160; nq and nk 1 .. 2^30.
 * Errors: INVALID_ARG (also: a zero or negative stride where none may be, scale not finite), ALIGNMENT, UNSUPPORTED, CUDA. */
dgq_status dgq_encoder_attn(const dgq_rows* Q, const dgq_rows* K, const dgq_rows* V, const dgq_rows* O, int dtype, int B,
                            int Hq, int Hkv, int nq, int nk, int d, float scale, const int32_t* kv_lens, void* stream);

/* A paged key/value cache in the caller's memory (codes 16-byte aligned).  Codes: dev int8 [n_pages, n_heads, page, row], row = d
 * rounded up to a multiple of 16; a value is code * scale with one fp32 scale for each page and head, dev [n_pages, n_heads].
 * page is 16, 32, 64 or 128; d a multiple of 8 up to 160; n_pages * page < 2^31.  Slot s is row s % page of page s / page. */
typedef struct {
  void *k, *v;
  float *k_scale, *v_scale;
  int n_pages, n_heads, page, d;
} dgq_kv_cache;

/* Block tables and slot maps from lengths.  B requests hold lens[b] tokens and get n_new[b] more (dev int32 [B]).  Entry i
 * of block_table[b] (dev int32 [B, max_pages]) is the page of tokens i * page .. : the pages that request b lacks are taken
 * from the front of free_pages (dev int32 [n_free]) in the order of the requests and entered behind those it has; other
 * entries stay as they are.  Written: token_start[B + 1] (prefix sums of n_new: where each request's rows begin in a
 * packed batch), kv_lens[B] = lens + n_new, slots[n_slots] (the slot of every new token in that order; -1 behind the last
 * one) and used[1] = free pages taken.
 * What does not fit is found on the device, which records DGQ_ERR_INVALID_ARG in the status word: negative lengths count
 * as 0, lengths beyond max_pages * page as that, a page that free_pages has no more entry for becomes -1, as do the slots of its
 * tokens, of tokens on a page that is negative or whose slots do not fit 31 bits, and of those beyond n_slots or the table.
 * The outputs may not overlap lens and n_new.  B is at least 1; each eight requests read all lengths, which is meant for thousands of
 * requests, not for millions.  Errors: INVALID_ARG, UNSUPPORTED (page), CUDA. */
dgq_status dgq_kv_plan(const int32_t* lens, const int32_t* n_new, int B, const int32_t* free_pages, int n_free,
                       int32_t* block_table, int max_pages, int page, int32_t* token_start, int32_t* kv_lens, int32_t* slots,
                       int n_slots, int32_t* used, void* stream);

/* Rows K[t], V[t] (t < T; [1, T, n_heads, d]) into slots[t] (dev int32 [T]; negative: the row is skipped).  The rows of one page
 * stand next to each other in ascending order, as dgq_kv_plan gives them; there may be rows of the page between them that get
 * nothing, and any number of skipped ones.  For each page and
 * head, in fp32: top = max |x| over the page's rows of this call, s = max(top * (1 / 127), 2^-126), 0 where top is 0; a page whose
 * row 0 is among them forgets what it held, any other one keeps its rows below the first new one: s = max(s, scale), and where s has
 * grown, their codes become rint((code * scale) / s).  New codes are rint(x / s), 0 where s is 0.  Each operation is rounded to
 * fp32, rint to the nearest whole number, ties to even.  Rows behind the first
 * new one that get nothing stay as they are.  A value that is not finite counts as 0 and is recorded as DGQ_ERR_INVALID_ARG in the
 * status word; rows that are skipped may hold anything.  A slot beyond the cache is skipped and recorded too, as is one that is not
 * above all of its page's before it.  Of a page whose rows stand in
 * several places of a call, with another page's rows between them, or to which two calls write at the same time, the codes and scales
 * are not defined afterwards.
 * Errors: INVALID_ARG, ALIGNMENT, UNSUPPORTED, CUDA. */
dgq_status dgq_kv_write(const dgq_kv_cache* cache, const dgq_rows* K, const dgq_rows* V, int dtype, int64_t T,
                        const int32_t* slots, void* stream);

/* The rows of slots[t] as the values they stand for, code * scale rounded to `dtype`, into K[t], V[t] ([1, T, n_heads, d]):
 * contiguous keys and values again, as dgq_cross_attn_logq takes them.  A negative slot gives zeros, one beyond the cache too
 * (and DGQ_ERR_INVALID_ARG in the status word).  Errors: as above. */
dgq_status dgq_kv_read(const dgq_kv_cache* cache, const int32_t* slots, int64_t T, const dgq_rows* K, const dgq_rows* V,
                       int dtype, void* stream);

/* Attention as in dgq_encoder_attn over the first kv_lens[b] tokens of each request's pages (block_table dev int32
 * [B, max_pages], kv_lens dev int32 [B]; lengths outside 0 .. max_pages * page are taken as the nearer end).
 * q_start NULL: Q, O [B, max_nq, Hq, d].  Else Q, O [1, n_rows, Hq, d] packed: request b has rows q_start[b] .. q_start[b + 1] - 1
 * (dev int32 [B + 1], ascending), at most max_nq of them; other rows of O stay as they are.  causal != 0: row i of n sees the first
 * kv_lens[b] - n + i + 1 tokens (the n queries belong to the last n tokens).  Hq a multiple of cache->n_heads.  Pages may be
 * shared by requests.  max_pages * page, max_nq and n_rows are at most 2^30.  Weights are rounded to fp16 for the product with the codes,
 * whatever `dtype` is.  The value scales of the pages that a row sees are within 2^80 of one another (a page of zeros counts as one of
 * 2^-40, scales below 2^-100 as 2^-100); a weight on a page of far smaller values than that would be lost from the row's sum.
 * Found on the device and recorded as DGQ_ERR_INVALID_ARG in the status word: table entries outside the cache (their tokens
 * count as absent), more than max_nq rows or rows beyond n_rows (left out).  n_rows is ignored where q_start is NULL.
 * Errors: INVALID_ARG, ALIGNMENT, UNSUPPORTED, CUDA. */
dgq_status dgq_cached_attn(const dgq_kv_cache* cache, const dgq_rows* Q, const dgq_rows* O, int dtype, int B, int Hq,
                           int64_t n_rows, const int32_t* q_start, int max_nq, const int32_t* block_table, int max_pages,
                           const int32_t* kv_lens, int causal, float scale, void* stream);

/* ---------------------------------------------------------------- group norm, and products of few rows with 4-bit weights
 * (What stands around the convolutions of a UNet's residual block; the paper leaves it in 16 bits.  The calls of this section are this
 * library's own.  dgq_group_norm, dgq_group_norm_quantize and dgq_linear_few only enqueue work on `stream`, allocate nothing and do
 * not synchronise.  Work goes to the current device, where all memory and objects have to be.) */

enum { DGQ_ACT_NONE = 0, DGQ_ACT_SILU = 1 }; /* SiLU: y / (1 + e^-y) */

/* Group norm of channels-last maps X [B, P, C] (P pixels; `head` of the strides is ignored) of type `dtype`, with an addend per
 * image and channel (dev [B, C] of the same type, rows ld_add elements apart, 0 for one that all images share; NULL: none):
 *   u = x + add[b, c];  y = (u - mean) / sqrt(var + eps) * gamma[c] + beta[c];  Y = act(y), rounded once,
 * mean and (biased) variance over the P pixels and C / n_groups neighbouring channels of a group.  gamma, beta: dev fp32 [C], NULL for 1
 * and 0.  Sums are held in 32 bits or more.  A group that holds a value that is not finite gives NaN.  (Of a y far
 * below nought a SiLU leaves up to 2^-60 |y|.)  Y may be X (the same pointer and strides); it may not overlap X otherwise.
 * C a multiple of 8 up to 4096, any n_groups that divides it, eps at least 2^-126.
 * workspace: dev, 256-byte aligned, at least dgq_group_norm_workspace_bytes(); contents undefined on entry and exit; calls that may
 * overlap on the GPU need separate ones.
 * Errors: INVALID_ARG (also: pixel rows of Y, of one image or of two, that overlap), ALIGNMENT, UNSUPPORTED (also: B > 65535, P > 2^30), WORKSPACE, CUDA. */
dgq_status dgq_group_norm(const dgq_rows* X, const void* add, int64_t ld_add, const float* gamma, const float* beta,
                          const dgq_rows* Y, int dtype, int B, int P, int C, int n_groups, float eps, int act, void* workspace,
                          size_t workspace_bytes, void* stream);
/* The same, straight into the codes of a layer: Xq dev bytes [B * P, K_pad] as dgq_quantize_act lays them out, with the static table
 * of `timestep` (row i = b * P + p is pixel position i mod the grouping's own P), C channels of the grouping.  The value that is
 * quantized is act(y) itself, not its rounding to 16 bits:
 *   q = clamp(rint(act(y) * inv_s) + Z, 0, 2^b - 1)   as 64-bit arithmetic on the 16-bit inputs gives it (inv_s is the table's fp32
 * number; var is a difference of 64-bit sums, off by 2^-50 of mean^2 + add^2): the codes do not depend on how the sums were split.  NaN gives code 0.
 * DGQ_CODES_S8_CENTRED has the limits of dgq_quantize_act.  Xq is 16-byte aligned and does not overlap X.  n_groups at most 2048.
 * Errors: as above, NOT_CALIBRATED, INVALID_ARG also for a grouping of another device than the current one. */
dgq_status dgq_group_norm_quantize(const dgq_groups* g, int timestep, int layout, const dgq_rows* X, const void* add,
                                   int64_t ld_add, const float* gamma, const float* beta, int dtype, int B, int P, int n_groups,
                                   float eps, int act, void* Xq, void* workspace, size_t workspace_bytes, void* stream);
/* Bytes for dgq_group_norm (quantize 0; 0 where the map is held on the chip: workspace may be NULL then) or dgq_group_norm_quantize. */
dgq_status dgq_group_norm_workspace_bytes(int B, int P, int C, int n_groups, int quantize, size_t* bytes);

/* A 4-bit weight whose scales each serve one output and `group` (32, 64 or 128) neighbouring input channels, for products with few
 * 16-bit rows (time embeddings, single tokens).  Library-owned; every call but _destroy synchronises with the host. */
typedef struct dgq_few_weight dgq_few_weight;
/* W dev fp16 [N, K], rounded to nearest: s = max |w| / 7 of the group rounded up to fp16, q = rint(w / s).  K a multiple of 8 (the last
 * group may be short), K and N up to 2^20 - 16.  Errors: INVALID_ARG (also: a weight that is not finite), UNSUPPORTED, CUDA. */
dgq_status dgq_few_weight_prepare(const void* W, int N, int K, int group, dgq_few_weight** out, void* stream);
/* The same from codes quantized elsewhere: wq dev int8 [N, K], -8 .. 7; scales dev fp16 [N, ceil(K / group)], finite.
 * Errors: INVALID_ARG (also: a code or scale outside these), UNSUPPORTED, CUDA. */
dgq_status dgq_few_weight_from_codes(const int8_t* wq, const void* scales, int N, int K, int group, dgq_few_weight** out,
                                     void* stream);
dgq_status dgq_few_weight_destroy(dgq_few_weight* w);
/* Host copies of the codes (int8 [N, K]) and of the scales' fp16 bits [N, ceil(K / group)]; either may be NULL. */
dgq_status dgq_few_weight_export(const dgq_few_weight* w, int8_t* wq, uint16_t* scales);
/* Y[m, n] = bias[n] + sum_g s[n, g] * sum over the channels k of group g of q[n, k] * act(X[m, k]), summed in fp32 and rounded once.
 * X dev [M, K], Y dev [M, N], bias dev [N] or NULL, all of type `dtype`; X 16-byte aligned, its rows ldx elements apart (a multiple of 8,
 * 0 allowed), those of Y ldy.  SiLU's results enter the product as two numbers of `dtype`, off by at most 2^-15 of them and 2^-119 (bf16), 2^-20 of
 * them and 2^-25 (fp16, whose second number is below the smallest normal one where the result is below 1/8).  A sum over a group's q and x that fp32 does
 * not hold is infinite.  Any M; the weight is read once for every 32 rows, so that for many rows dgq_linear is the better call.
 * Errors: INVALID_ARG (also: a weight of another device than the current one), ALIGNMENT, UNSUPPORTED (M > 2^21 - 32), CUDA. */
dgq_status dgq_linear_few(const dgq_few_weight* w, const void* X, int64_t ldx, int dtype, int M, int act, const void* bias, void* Y,
                          int64_t ldy, void* stream);

/* ---------------------------------------------------------------- cross-attention without a caller workspace
 * (The paper has no counterpart: this is a deployment convenience of this library.)
 * Same computation, arguments and results as dgq_cross_attn_logq, for callers that
 * have no way to obtain device memory for the workspace: code running inside a
 * region where allocation is forbidden (a plugin or runtime callback that is only
 * handed its input and output buffers, a real-time loop that must not call the
 * allocator, a host that has already committed all device memory).  The scratch
 * space lives in a fixed array inside the library image instead:
 *   - DGQ_NOALLOC_SCRATCH_BYTES of device memory are held by every GPU that loads
 *     the library, from load until the process exits, whether or not this call is
 *     ever used;
 *   - the problem must satisfy B * H * nq <= DGQ_NOALLOC_MAX_ROWS and
 *     B * H <= DGQ_NOALLOC_MAX_HEADS, else DGQ_ERR_WORKSPACE is returned and
 *     nothing is launched;
 *   - the first call on each device looks up the device address of the array
 *     (with that device current) and remembers it; make that first call before
 *     starting any stream capture.  Later calls only enqueue work on `stream`;
 *   - the call itself performs no allocation and frees nothing;
 *   - all calls on a device share the one array.  It still holds the previous
 *     call's statistics on entry; nothing in it has to start clean, because the
 *     first kernel writes every entry that the second one reads.  Two calls whose
 *     kernels can overlap on the GPU (different streams without an ordering
 *     between them) race on it:
 *     serialise them, or use dgq_cross_attn_logq with separate workspaces.
 * Errors: those of dgq_cross_attn_logq, checked first and in the same order; then
 * DGQ_ERR_WORKSPACE for a problem beyond the limits above; DGQ_ERR_UNSUPPORTED when
 * the current device's ordinal is 64 or more (the library remembers one address per
 * device ordinal below that). */
#define DGQ_NOALLOC_MAX_ROWS (1 << 18)
#define DGQ_NOALLOC_MAX_HEADS 256
#define DGQ_NOALLOC_SCRATCH_BYTES (4 * (DGQ_NOALLOC_MAX_ROWS / 128 + DGQ_NOALLOC_MAX_HEADS) + 8 * DGQ_NOALLOC_MAX_ROWS)
dgq_status dgq_cross_attn_logq_noalloc(const void* Q, const void* K, const void* V, int B, int H, int nq, int nk,
                                       int d, int score_bits, int scale_gran, const float* fixed_scale, void* O,
                                       float* scale_out, uint8_t* codes_out, void* stream);

/* ---------------------------------------------------------------- status
 * Synchronises the current device and returns the device status word of the
 * current device in *status (DGQ_OK, or the first error a kernel recorded),
 * then clears it. */
dgq_status dgq_device_status(int* status);
/* Diagnostic: enqueues a kernel that runs each of the library's bounded waits on a barrier nobody arrives at, with a
 * limit of max_polls (1..65536) times 1024 SM clocks (about half a microsecond each) in place of the usual second, so
 * that the time-out path of the bounded waits (other waits of the block end too, status word, dgq_device_status, a
 * usable device afterwards) can be exercised without making a wait of a working kernel run out.
 * Errors: INVALID_ARG, CUDA. */
dgq_status dgq_selftest_wait_timeout(uint32_t max_polls, void* stream);
const char* dgq_status_string(dgq_status s);
/* Number of kernels the library has launched in this process (all devices). */
uint64_t dgq_launch_count(void);

#ifdef __cplusplus
}
#endif
#endif /* DGQ_H_ */
