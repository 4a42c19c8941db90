/*
 * ditmi.h -- C ABI of the MI355X (gfx950) DiT denoising-step library.
 *
 * The library computes the Diffusion Transformer stage of an
 * Encoder -> DiT -> Decoder generation pipeline: the stage that iteratively
 * denoises the latent and dominates serving time (paper: Background and
 * Motivation, "Diffusion Model Architecture" and "Workload Characteristics";
 * System Design, the Transformer service that runs the denoising backbone and
 * updates the latent).  The paper does not write the block out; the block
 * computed is the adaLN-Zero DiT block of the work the paper cites for this
 * stage (Peebles & Xie, arXiv:2212.09748):
 *
 *   (shift1, scale1, gate1, shift2, scale2, gate2) = SiLU(c) W_ada^T + b_ada
 *   x1 = x  + gate1 * (Attn(LN(x) * (1 + scale1) + shift1) W_o^T + b_o)
 *   y  = x1 + gate2 * (GELU_tanh((LN(x1) * (1 + scale2) + shift2) W_1^T + b_1) W_2^T + b_2)
 *
 * LN has no affine, biased variance, eps = shape.ln_eps.  Attn is full
 * bidirectional multi-head attention with scale 1/sqrt(head_dim); the QKV
 * projection's output column j is s*hidden + head*head_dim + d, s in (q,k,v).
 * With text_tokens > 0 the block is the joint two-stream block: image and
 * text tokens each use their own weights (same c) and attention runs over
 * the concatenation [image; text].
 *
 * Conventions for every entry point:
 *   - Pointers to tensors are DEVICE pointers, 16-byte aligned, owned by the
 *     caller; the library never allocates or frees device memory while
 *     computing.  Its only device state is the static scratch array of
 *     dit_block_forward_noalloc (below), which lives until the process ends.
 *   - Weight matrices are row-major [out, in]; weights and biases have the
 *     element type shape.dtype (fp32 or bf16).  Residual streams, the
 *     conditioning vector, patches and outputs are always fp32.
 *   - Work is enqueued on `stream` (a hipStream_t; NULL = the default
 *     stream) and the call returns without synchronising.
 *   - All arguments are validated before anything is enqueued: a call that
 *     returns an error has enqueued no work.  NaN/Inf inputs are not errors;
 *     they propagate.  No call aborts or throws.
 *   - dit_last_error() returns the text of the calling thread's last failure.
 *   - Calls are thread-safe; concurrent calls must not share a workspace.
 *   - Every kernel of a call runs on `stream`; the library creates no
 *     streams.  No allocation or memset is enqueued by any call, so the
 *     calls can be captured into a HIP graph.
 *   - Size limits (DIT_ERR_UNSUPPORTED beyond them): rows = B * (T + Tt)
 *     below 2^24 with rows * max(3D, F) below 2^31, and every weight matrix
 *     (in particular F * D) below 2^31 elements: element indices fit 32 bits,
 *     and so do the byte offsets of bf16 operands (fp32 operands, up to 8 GiB,
 *     are addressed with 64 bits).
 */
#ifndef DITMI_H
#define DITMI_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define DITMI_VERSION 1

typedef enum {
  DIT_OK = 0,
  DIT_ERR_INVALID_ARG = -1,  /* null pointer, bad size, misaligned pointer   */
  DIT_ERR_UNSUPPORTED = -2,  /* valid shape this library does not implement  */
  DIT_ERR_WORKSPACE = -3,    /* workspace smaller than dit_workspace_bytes()  */
  DIT_ERR_HIP = -4           /* a HIP runtime call or launch failed           */
} dit_status;

typedef enum { DIT_F32 = 0, DIT_BF16 = 1 } dit_dtype;

/* Workspace kinds for dit_workspace_bytes(). */
typedef enum { DIT_WS_BLOCK = 0, DIT_WS_STEP = 1, DIT_WS_COND = 2, DIT_WS_SAMPLE = 3, DIT_WS_SERVE = 4 } dit_ws_kind;

/* Shape of one DiT model / workload.
 *   batch         B >= 1 samples
 *   tokens        T >= 1 image (latent patch) tokens per sample
 *   text_tokens   Tt >= 0 text tokens per sample; > 0 selects the joint block
 *   hidden        D, multiple of 64, <= 4096
 *   heads, head_dim  heads * head_dim == hidden; head_dim in {64, 72, 128}
 *   mlp_hidden    F, multiple of 64
 *   n_blocks      L >= 1 (used by the step)
 *   patch_in      p*p*C channels of one latent patch (step), 1..256
 *   patch_out     channels predicted per token by the final layer (step), a
 *                 multiple of 4 in 4..256
 *   dtype         dit_dtype of weights and GEMM operands
 *   ln_eps        LayerNorm epsilon (> 0) */
typedef struct {
  int32_t batch, tokens, text_tokens;
  int32_t hidden, heads, head_dim, mlp_hidden, n_blocks;
  int32_t patch_in, patch_out;
  int32_t dtype;
  float ln_eps;
} dit_shape;

/* Weights of one stream of one block (device pointers, [out, in] row-major):
 *   w_ada [6D, D], b_ada [6D]   chunks (shift1, scale1, gate1, shift2, scale2, gate2)
 *   w_qkv [3D, D], b_qkv [3D]
 *   w_o   [D, D],  b_o   [D]
 *   w_fc1 [F, D],  b_fc1 [F]
 *   w_fc2 [D, F],  b_fc2 [D] */
typedef struct {
  const void *w_ada, *b_ada, *w_qkv, *b_qkv, *w_o, *b_o, *w_fc1, *b_fc1, *w_fc2, *b_fc2;
} dit_stream_weights;

/* txt is read only when shape.text_tokens > 0. */
typedef struct {
  dit_stream_weights img, txt;
} dit_block_weights;

/* Step weights.  `blocks` is a HOST array of n_blocks structs holding device
 * pointers.  w_patch [D, patch_in], b_patch [D]; pos [T, D] fp32 or NULL
 * (added after the patch embedding); w_ada_final [2D, D], b_ada_final [2D]
 * (chunks shift, scale); w_final [patch_out, D], b_final [patch_out]. */
typedef struct {
  const void *w_patch, *b_patch;
  const float *pos;
  const dit_block_weights *blocks;
  const void *w_ada_final, *b_ada_final, *w_final, *b_final;
} dit_step_weights;

/* Bytes of workspace the given kind of call needs for this shape (0 when the
 * shape is invalid; dit_last_error() then says why).  The workspace is device
 * memory owned by the caller, 256-byte aligned, contents need not be
 * initialised and are undefined after the call. */
size_t dit_workspace_bytes(const dit_shape *s, int kind);

/* One DiT block, in place (the unit of the DiT stage's per-step work).
 *   x      [B, T, D] fp32 image/latent residual stream, updated in place
 *   x_txt  [B, Tt, D] fp32 text residual stream, updated in place (joint
 *          block only; must be NULL when text_tokens == 0)
 *   cond   [B, D] fp32 conditioning vector c
 *   workspace  >= dit_workspace_bytes(s, DIT_WS_BLOCK) bytes
 * Errors: DIT_ERR_INVALID_ARG, DIT_ERR_UNSUPPORTED, DIT_ERR_WORKSPACE, DIT_ERR_HIP. */
dit_status dit_block_forward(const dit_shape *s, const dit_block_weights *w, float *x, float *x_txt,
                             const float *cond, void *workspace, size_t ws_bytes, void *stream);

/* Size of the static device scratch of dit_block_forward_noalloc (128 MiB
 * per GPU): enough for one block of DiT-XL/2 at 256 tokens x 8 samples
 * (42 MiB) or 1024 tokens x 4 (83 MiB). */
#define DIT_NOALLOC_SCRATCH_BYTES (128u << 20)

/* dit_block_forward for callers that cannot allocate device memory: code
 * being captured into a HIP graph, tight serving loops, harnesses that
 * forbid hipMalloc.  Same arguments, results and errors as
 * dit_block_forward, but the workspace is a static device array of
 * DIT_NOALLOC_SCRATCH_BYTES that the library holds on each GPU it runs on
 * until the process ends; the call allocates nothing and calls no
 * allocating library routine.  The GPU is the one `stream` belongs to (the
 * current device for NULL).  Its first call on a GPU looks the array's
 * device address up (hipGetSymbolAddress) and keeps it.
 * Every call on one GPU shares that GPU's array: calls that may overlap on
 * one GPU (different streams without ordering between them) race and give
 * undefined results; calls ordered on one stream are safe.  The array keeps
 * the last call's contents; nothing in it needs clearing.
 * Errors: those of dit_block_forward, and DIT_ERR_UNSUPPORTED when
 * dit_workspace_bytes(s, DIT_WS_BLOCK) exceeds DIT_NOALLOC_SCRATCH_BYTES
 * (checked before anything is enqueued). */
dit_status dit_block_forward_noalloc(const dit_shape *s, const dit_block_weights *w, float *x, float *x_txt,
                                     const float *cond, void *stream);

/* One denoising step: the full DiT forward of the paper's per-step DiT time
 * (paper Table: per-stage execution time; one step = one DiT forward):
 *   x = patches W_patch^T + b_patch (+ pos);  L blocks;
 *   out = (LN(x) * (1 + scale_f) + shift_f) W_final^T + b_final
 *   patches [B, T, patch_in] fp32;  out [B, T, patch_out] fp32 (may not alias)
 *   x_txt   [B, Tt, D] fp32 text stream, updated in place (joint only, else NULL)
 *   cond    [B, D] fp32
 *   workspace >= dit_workspace_bytes(s, DIT_WS_STEP) bytes
 * No sampler update is applied. */
dit_status dit_step_forward(const dit_shape *s, const dit_step_weights *w, const float *patches,
                            float *x_txt, const float *cond, float *out, void *workspace, size_t ws_bytes,
                            void *stream);

/* Timestep + class conditioning of class-conditional DiT (the work the paper
 * cites for the DiT stage):
 *   e = [cos(t f), sin(t f)], f_i = 10000^(-i/128), i < 128   (256 features)
 *   cond = (SiLU(e W_t1^T + b_t1)) W_t2^T + b_t2 + class_table[y]
 *   t [B] fp32 timesteps, y [B] int32 labels (0 <= y < n_rows of class_table,
 *   not checked on device); w_t1 [D, 256], b_t1 [D], w_t2 [D, D], b_t2 [D],
 *   class_table [*, D] in shape.dtype; cond [B, D] fp32 output.
 *   workspace >= dit_workspace_bytes(s, DIT_WS_COND) bytes. */
dit_status dit_cond_embed(const dit_shape *s, const float *t, const int32_t *y, const void *w_t1,
                          const void *b_t1, const void *w_t2, const void *b_t2, const void *class_table,
                          float *cond, void *workspace, size_t ws_bytes, void *stream);

/* Weights of the timestep + class conditioning (see dit_cond_embed). */
typedef struct {
  const void *w_t1, *b_t1, *w_t2, *b_t2, *class_table;
} dit_cond_weights;

/* The DiT stage's multi-step denoising loop (paper: Background and
 * Motivation, Workload Characteristics -- 40-50 iterations for standard
 * samplers, 4 or 8 for distilled ones; System Design -- the Transformer
 * service iterates the backbone over the timesteps and updates the latent).
 * The paper names no sampler; this is first-order Euler on the
 * flow-matching ODE in the patchified latent space:
 *   for i in 0 .. n_steps-1:
 *     c_i = cond_w ? class conditioning at t_i = (float)(sigmas[i] * t_scale)
 *                    and labels y (as dit_cond_embed)
 *                  : cond (the same for every step)
 *     v_i = one step (dit_step_forward) on z with c_i; joint models start every
 *           step from the given text states x_txt (which are not modified)
 *     z  += (sigmas[i+1] - sigmas[i]) * v_i      (difference taken in fp32)
 *   z       [B, T, P] fp32, P = patch_in = patch_out, updated in place
 *   sigmas  HOST array of n_steps + 1 floats (any order); n_steps >= 0
 *   cond_w  conditioning weights (class-conditioned models) with y [B] int32
 *           device labels, or NULL with cond [B, D] fp32 given
 *   x_txt   [B, Tt, D] fp32 text states (joint only, else NULL), read only
 *   workspace >= dit_workspace_bytes(s, DIT_WS_SAMPLE) bytes
 * Enqueues no allocation or memset, so the whole loop can be captured into a
 * HIP graph and replayed.  Errors as dit_step_forward. */
dit_status dit_sample_euler(const dit_shape *s, const dit_step_weights *w, const dit_cond_weights *cond_w,
                            const int32_t *y, const float *cond, const float *sigmas, int32_t n_steps,
                            float t_scale, float *z, const float *x_txt, void *workspace, size_t ws_bytes,
                            void *stream);

/* One request handed to the DiT stage: host buffers (page-locked for the
 * copies to overlap; pageable memory works but serialises) of the latent from
 * the encoder stage, the denoised latent for the decoder stage, and the
 * request's conditioning input. */
typedef struct {
  const float *z_in;      /* [B, T, P] fp32 */
  float *z_out;           /* [B, T, P] fp32 */
  const int32_t *y;       /* [B] labels when conditioning weights are given, else NULL */
  const float *cond;      /* [B, D] fp32 conditioning otherwise, else NULL */
} dit_request;

/* Serve a sequence of requests through the DiT stage on one GPU: the paper's
 * asynchronous inter-stage pipeline (System Design: the stages communicate
 * through asynchronous queues so that requests occupy different stages at
 * once; Challenge 1: asynchronous handoff absorbs transfer jitter) shrunk to
 * one device.  Per request: copy z_in (and y or cond) host -> device, run the
 * Euler loop of dit_sample_euler (same sigmas, n_steps, t_scale for every
 * request), copy the result device -> host into z_out.
 *   overlap != 0: the copies run on copy_stream (required) and the loops on
 *     `stream`, with two device slots ordered by events: the input of request
 *     i+1 and the output of request i-1 move while request i computes.
 *   overlap == 0: everything runs in order on `stream`.
 *   jitter_us > 0: before enqueueing each request the calling thread sleeps a
 *     pseudo-random time in [0, jitter_us] microseconds (seeded by
 *     jitter_seed), standing in for irregular arrivals from the encoder
 *     stage; results do not depend on it.
 * Results are identical for every overlap/jitter setting.  The call returns
 * after enqueueing; synchronise `stream` before reading z_out.  Temporary
 * HIP events are created and released by the call (no device memory).
 *   workspace >= dit_workspace_bytes(s, DIT_WS_SERVE) bytes */
dit_status dit_serve(const dit_shape *s, const dit_step_weights *w, const dit_cond_weights *cond_w,
                     const dit_request *reqs, int32_t n_requests, const float *sigmas, int32_t n_steps,
                     float t_scale, int32_t overlap, uint32_t jitter_us, uint32_t jitter_seed, void *workspace,
                     size_t ws_bytes, void *stream, void *copy_stream);

/* Fixed 2-D sin-cos position table of DiT, pos [grid_h*grid_w, hidden] fp32,
 * token n = r*grid_w + c: features [0, D/2) encode column c, [D/2, D) row r;
 * each half is [sin(p w_i), cos(p w_i)], w_i = 10000^(-i/(D/4)).
 * hidden must be a multiple of 4. */
dit_status dit_pos_embed_2d(int32_t grid_h, int32_t grid_w, int32_t hidden, float *pos, void *stream);

/* ------------------------------------------------------------------------
 * Stand-alone operators.  The conventions above hold: device pointers, the
 * caller's workspace and stream, everything checked before the first launch,
 * no allocation, no atomics, results that do not depend on earlier calls.
 * What the host cannot see (the int32 index arrays on the device) is bounded
 * by the kernels: an entry out of range is clamped into it, so such a call
 * computes something useless but stays inside the tensors.  Outputs must not
 * overlap inputs unless said otherwise, nor one another.
 * ------------------------------------------------------------------------ */

/* Masked attention over documents (requests, samples): packed one behind the
 * other in one sequence, padded to equal rooms, or single new tokens over the
 * rooms of a cache.  The block's own attention knows one length per batch and
 * no mask; this is the attention of a batch of mixed resolutions, of padded
 * text, of prefix-conditioned generation.
 *
 * Document d has query rows q_start[d] .. q_start[d+1]-1 (nq of them) of q
 * and o, and key rows k_start[d] .. k_start[d]+nk-1 of k and v, with
 * nk = min(k_len[d], k_start[d+1] - k_start[d]).  For its query i, key j and
 * head h (keys of head h / (heads / kv_heads)):
 *   s = scale * q.k
 *   s = cap * tanh(s / cap)                     where cap > 0
 *   s = s - slopes[h] * |i + nk - nq - j|       where slopes is given
 *   j is visible when j < nk and
 *     DIT_MASK_FULL    always
 *     DIT_MASK_CAUSAL  j <= i + nk - nq         (the last query sees every key)
 *     DIT_MASK_PREFIX  j <= i + nk - nq or j < prefix[d]
 *   o = softmax over the visible keys of s, times v
 * A query without a visible key gets zeros.  What k and v hold in rows that a
 * query cannot see (NaN and infinities included) does not reach it; a value that
 * it sees and that is not finite leaves nothing finite in its column.  A score
 * of -inf gives its key the weight 0, and a query that has no other zeros (with
 * a cap, an infinite q.k is a score of -cap or cap).  Rows of o outside every
 * document are left as they were.  fp32 softmax and sums; in bf16 the probabilities, taken
 * relative to a running maximum, are rounded to bf16 before the product with
 * v, and their sum is that of the rounded ones.  No probability exceeds 1, and
 * they are added up before the division by their sum: finite values of v give
 * finite results as long as the largest times the number of visible keys stays
 * below 2^127.
 *   docs >= 1;  heads a multiple of kv_heads;  head_dim in {64, 72, 128}
 *   q_rows, k_rows   rows of q and o, rows of k and v (every room counted)
 *   max_q, max_k     no document has more query rows, or keys (longer ones
 *                    are cut to them)
 *   dtype            of q, k, v and o
 *   scale > 0 (at most 2^100);  cap 0 (none) or in 2^-20 .. 2^12
 *   *_row, *_head    strides in elements between rows and between heads of
 *                    each tensor, multiples of 8 (bf16) or 4 (fp32); the
 *                    head_dim elements of a head are contiguous.  Rows at
 *                    most 2^22 elements apart.  No two pieces (row, head) of
 *                    o may share elements. */
typedef enum { DIT_MASK_FULL = 0, DIT_MASK_CAUSAL = 1, DIT_MASK_PREFIX = 2 } dit_attn_mask;
typedef struct {
  int32_t docs, heads, kv_heads, head_dim;
  int32_t q_rows, k_rows, max_q, max_k;
  int32_t dtype, mask;
  float scale, cap;
  int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head;
} dit_attn_shape;

/* Bytes of workspace of dit_attention (it may be 0: then pass NULL); -1 cast
 * to size_t for an invalid shape, dit_last_error() then says why. */
size_t dit_attention_workspace_bytes(const dit_attn_shape *s);

/*   q_start, k_start  [docs + 1] int32, not falling, or NULL for equal rooms of
 *                     max_q query rows (max_k key rows) each.  (Of a q_start
 *                     that falls, documents may share query rows; each such row
 *                     of o then holds pieces of their results.)
 *   k_len             [docs] int32 filled keys of each document, or NULL: all
 *   prefix            [docs] int32 (DIT_MASK_PREFIX; NULL otherwise)
 *   slopes            [heads] fp32, or NULL
 *   workspace         256-byte aligned */
dit_status dit_attention(const dit_attn_shape *s, const void *q, const void *k, const void *v, void *o,
                         const int32_t *q_start, const int32_t *k_start, const int32_t *k_len,
                         const int32_t *prefix, const float *slopes, void *workspace, size_t ws_bytes,
                         void *stream);

/* 8-bit floating point (OCP e4m3: 448 the largest value, no infinities) with
 * an fp32 scale for every block of 128 columns, of one row (block_rows = 1:
 * activations) or of 128 rows (block_rows = 128: weights):
 *   scale = max(amax * (1 / 448), 2^-126),  code = e4m3(x * (1 / scale))
 * rounded to nearest even; the last blocks of a row or a column may be
 * partial.  NaN becomes the NaN code, in a block whose scale comes from its
 * other values; an infinity makes its block's scale infinite.
 *   x      [rows, cols] of dtype (fp32 or bf16), rows x_row elements apart
 *   codes  [rows, cols] bytes, contiguous
 *   scale  [ceil(rows / block_rows), ceil(cols / 128)] fp32
 *   cols, x_row: multiples of 8;  rows >= 0 */
dit_status dit_quantize_fp8(int32_t rows, int32_t cols, int32_t block_rows, int32_t dtype, const void *x,
                            int64_t x_row, void *codes, float *scale, void *stream);

/* A linear layer on such operands:
 *   y[m, n] = act(sum_k a[m, k] a_scale[m, k/128] * w[n, k] w_scale[n/128, k/128] + bias[n])
 * A block's products are added before they are scaled: for an fp32 output in
 * fp32, otherwise on the 8-bit matrix pipe, which adds every 8 consecutive
 * products aligned to the largest of them with a last place of 2^-13 of its
 * binade, and those sums in fp32.
 *   rows >= 0, in a multiple of 16, out >= 1
 *   act    DIT_ACT_NONE, DIT_ACT_GELU (tanh)
 *   dtype  of out: DIT_F32, DIT_BF16, or DIT_E4M3, which quantises every row
 *          of y anew in blocks of 128 (as dit_quantize_fp8 with block_rows 1)
 *          into out and out_scale [rows, ceil(out / 128)] */
#define DIT_E4M3 2
typedef enum { DIT_ACT_NONE = 0, DIT_ACT_GELU = 1 } dit_activation;
typedef struct {
  int32_t rows, in, out;
  int32_t act, dtype;
} dit_linear_shape;

/* As dit_attention_workspace_bytes. */
size_t dit_linear_fp8_workspace_bytes(const dit_linear_shape *s);

/*   a [rows, in], w [out, in] e4m3 codes; a_scale [rows, ceil(in / 128)],
 *   w_scale [ceil(out / 128), ceil(in / 128)] fp32; bias [out] or NULL (fp32
 *   for DIT_F32, else bf16); out [rows, out]; out_scale for DIT_E4M3, else
 *   NULL.  All contiguous. */
dit_status dit_linear_fp8(const dit_linear_shape *s, const void *a, const float *a_scale, const void *w,
                          const float *w_scale, const void *bias, void *out, float *out_scale, void *workspace,
                          size_t ws_bytes, void *stream);

/* The norms around a sub-layer with its gate and residual, in one pass (the
 * block with norms before and after each sub-layer):
 *   x_out = res_scale * x + gate_b * (norm_post(y) * w_post)
 *   h     = norm_pre(x_out) * w_pre * (1 + scale_b) + shift_b
 * DIT_NORM_LAYER subtracts the mean and divides by the standard deviation
 * (biased variance), DIT_NORM_RMS divides by the root mean square, both with
 * eps; DIT_NORM_NONE (post only) leaves y as it is.  b = row_batch[row].
 *   rows >= 0 (at most 2^25; 2^24 - 1 of more than 4096 columns), hidden a
 *              multiple of 8 in 8 .. 8192
 *   batch      rows of gate, shift and scale, mod_stride elements apart (a
 *              multiple of 4): slices of one modulation matrix
 *   y_dtype    of y: DIT_F32 or DIT_BF16
 *   h_dtype    of h: DIT_F32, DIT_BF16 or DIT_E4M3 (with h_scale
 *              [rows, ceil(hidden / 128)], as dit_quantize_fp8, block_rows 1)
 *   x, x_out   [rows, hidden] fp32; x_out may be x itself
 *   y          [rows, hidden], or NULL: x_out = res_scale * x (x_out may be
 *              NULL too: then h is the norm of res_scale * x alone)
 *   h          [rows, hidden], or NULL: no norm follows
 *   w_post, w_pre  [hidden] fp32 or NULL (ones);  gate NULL: ones;
 *   shift, scale   both or neither;  row_batch [rows] int32, or NULL: equal
 *              samples of rows / batch rows each (rounded up) */
typedef enum { DIT_NORM_NONE = 0, DIT_NORM_LAYER = 1, DIT_NORM_RMS = 2 } dit_norm_kind;
typedef struct {
  int32_t rows, hidden, batch;
  int32_t post, pre;
  int32_t y_dtype, h_dtype;
  float eps, res_scale;
  int64_t mod_stride;
} dit_norm_shape;
dit_status dit_norm_residual(const dit_norm_shape *s, const float *x, float *x_out, const void *y,
                             const float *w_post, const float *gate, const float *w_pre, const float *shift,
                             const float *scale, const int32_t *row_batch, void *h, float *h_scale, void *stream);

/* Queries and keys between their projection and attention, in one pass: every
 * head normed on its own and turned by the positions of its row (a rotation of
 * pairs of its elements: rows and columns of an image; frames, rows and columns
 * of a video; one axis of text).  For row r, head h and x = q or k:
 *   n = norm(x) * w                     (DIT_NORM_LAYER, DIT_NORM_RMS with eps, as
 *                                       dit_norm_residual, over head_dim; or NONE)
 *   t = pos[r, axis of p] * freqs[p]    (radians; reduced to one turn in 64 bits)
 *   (n_a, n_b) = (n_a cos t - n_b sin t, n_a sin t + n_b cos t)    for pair p
 * Pair p are the elements (2p, 2p + 1) with DIT_PAIR_NEIGHBOURS and (p, p + P) with
 * DIT_PAIR_HALVES, P the number of all pairs; the first pairs[0] belong to axis 0,
 * the next pairs[1] to axis 1 and so on.  Elements from 2P on are not turned.
 * Statistics, weights and rotation in fp32 (for DIT_BF16 with cosines and sines that
 * are off by 2^-18 at most), one rounding at the end; the squares of a head must not
 * overflow fp32.
 * Row r of q goes to row q_dst[r] of q_out (r itself without q_dst), row r of k and
 * of v, which is copied as it is, to row k_dst[r] of k_out and v_out: the rooms of
 * a cache, or a joint sequence.  A row whose destination lies outside of the output
 * is not written; of two rows with one destination either's pieces may stay.  Other
 * rows of the outputs are left as they were.  q_out may be q itself (k_out k, v_out
 * v), with the same strides and without q_dst (k_dst); an output that shares some
 * elements with a tensor at another offset is one that overlaps it, and is not refused.
 *   rows >= 0 (at most 2^24);  heads, kv_heads >= 0 (at most 65535; either may be
 *              0: then its tensors are not read and may be NULL);  head_dim a
 *              multiple of 8 in 8 .. 256
 *   q_out_rows, k_out_rows   rows of q_out; of k_out and v_out
 *   dtype      of q, k, v and the outputs: DIT_F32 or DIT_BF16
 *   axes       0 .. 4;  pairs of each, together at most head_dim / 2 (a multiple of
 *              4 with DIT_PAIR_HALVES)
 *   eps        at least 2^-126
 *   *_row, *_head   strides as in dit_attn_shape */
typedef enum { DIT_PAIR_NEIGHBOURS = 0, DIT_PAIR_HALVES = 1 } dit_pairing;
typedef struct {
  int32_t rows, heads, kv_heads, head_dim;
  int32_t q_out_rows, k_out_rows;
  int32_t dtype, norm, pairing, axes;
  int32_t pairs[4];
  float eps;
  int64_t q_row, q_head, k_row, k_head, v_row, v_head;
  int64_t q_out_row, q_out_head, k_out_row, k_out_head, v_out_row, v_out_head;
} dit_qk_shape;

/*   v, v_out   both or neither (one without rows may be NULL beside the other)
 *   w_q, w_k   [head_dim] fp32 or NULL (ones)
 *   pos        [rows, axes] int32;  freqs [P] fp64 (both NULL without pairs)
 *   q_dst, k_dst   [rows] int32 or NULL */
dit_status dit_qk_norm_rope(const dit_qk_shape *s, const void *q, const void *k, const void *v, void *q_out, void *k_out,
                            void *v_out, const float *w_q, const float *w_k, const int32_t *pos, const double *freqs,
                            const int32_t *q_dst, const int32_t *k_dst, void *stream);

/* Microscaled 4-bit floating point (OCP MXFP4: e2m1 codes of 0, 0.5, 1, 1.5, 2, 3,
 * 4, 6 and their negatives, a power of two for every 32 columns of a row):
 *   scale = the least 2^e, e >= -127, with amax / scale < 7
 *   code  = e2m1(x / scale), to nearest, ties to even
 * so that the largest value rounds to 6 at most and none is off by more than half
 * a step.  A NaN or an infinity makes its block's scale the stored value 255, which
 * is not a number.
 *   x      [rows, cols] of dtype (fp32 or bf16), rows x_row elements apart
 *   codes  [rows, cols / 2] bytes, the even column in the lower four bits, contiguous
 *   scale  [ceil(cols / 256), rows, 8] bytes e + 127 (e8m0), contiguous: block b of
 *          row r at [b / 8, r, b % 8], so that what a tile of a product reads at
 *          once lies together; 0 behind the last column
 *   cols   a multiple of 32 (at most 2^30);  x_row a multiple of 8, >= cols (at most
 *          2^40);  rows >= 0, fewer than 2^24 pieces of 8 rows of 256 columns */
dit_status dit_quantize_fp4(int32_t rows, int32_t cols, int32_t dtype, const void *x, int64_t x_row, void *codes, void *scale,
                            void *stream);

/* The values of such codes and scales, x = code * scale (exact in fp32, and in bf16
 * where it has them; past the largest of x's type an infinity). */
dit_status dit_dequantize_fp4(int32_t rows, int32_t cols, int32_t dtype, const void *codes, const void *scale, void *x,
                              int64_t x_row, void *stream);

/* A linear layer on such operands:
 *   y[m, n] = act(sum_k a[m, k] a_scale[m, k/32] * w[n, k] w_scale[n, k/32] + bias[n])
 * with products and their sums in fp32 on the 4-bit matrix pipe.
 *   rows >= 0 (at most 2^26), in a multiple of 32 (at most 2^22), out >= 1 (at most
 *          2^26), and a grid of fewer than 2^32 threads
 *   act    as dit_linear_fp8
 *   dtype  of out: DIT_F32, DIT_BF16, or DIT_MXFP4, which quantises every row of y
 *          anew (as dit_quantize_fp4) into out and out_scale; out a multiple of 32 */
#define DIT_MXFP4 3
size_t dit_linear_fp4_workspace_bytes(const dit_linear_shape *s);

/*   a [rows, in / 2], w [out, in / 2] codes; a_scale [ceil(in / 256), rows, 8],
 *   w_scale [ceil(in / 256), out, 8]; bias [out] or NULL (fp32 for DIT_F32, else
 *   bf16); out [rows, out] ([rows, out / 2] codes for DIT_MXFP4); out_scale
 *   [ceil(out / 256), rows, 8] for DIT_MXFP4, else NULL.  All contiguous.  Scales
 *   behind the last column of an operand are not used. */
dit_status dit_linear_fp4(const dit_linear_shape *s, const void *a, const void *a_scale, const void *w, const void *w_scale,
                          const void *bias, void *out, void *out_scale, void *workspace, size_t ws_bytes, void *stream);

/* Kernel timing hook for measurement.  dit_timing_enable() (host allocation
 * of HIP events, not a compute call) makes every later launch of kernel class
 * `kclass` record a start/stop hipEvent pair on its launch stream (timing-only
 * events, created without the system-scope fence), for up to max_launches
 * launches, and accumulates the algorithmic flops and bytes of
 * those launches.  dit_timing_read() synchronises on the recorded events and
 * returns the sum of launch durations (ms), the number of launches, and the
 * algorithmic flop and byte totals.  dit_timing_disable() frees the events. */
typedef enum {
  DIT_K_GEMM_QKV = 0, DIT_K_ATTENTION = 1, DIT_K_GEMM_OUT = 2, DIT_K_GEMM_FC1 = 3,
  DIT_K_GEMM_FC2 = 4, DIT_K_LN_MOD = 5, DIT_K_ADALN = 6, DIT_K_OTHER = 7, DIT_K_COUNT = 8
} dit_kernel_class;
dit_status dit_timing_enable(int kclass, int max_launches);
dit_status dit_timing_read(double *total_ms, int *launches, double *flops, double *bytes);
dit_status dit_timing_disable(void);

const char *dit_status_string(dit_status st);
const char *dit_last_error(void);
int dit_version(void);

#ifdef __cplusplus
}
#endif
#endif /* DITMI_H */
