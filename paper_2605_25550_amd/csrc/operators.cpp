// Host side of the stand-alone operators: argument validation, workspace
// sizes and launches.  Every argument is checked before the first launch.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "host.h"
#include "kernels.h"

using namespace ditmi;

namespace {

constexpr size_t BAD_SIZE = (size_t)-1;

// ------------------------------------------------------------------ attention
dit_status check_strides(const char* name, int64_t row, int64_t head, int heads, int rows, int dh, int unit) {
  if (row < 0 || head < 0 || row % unit != 0 || head % unit != 0)
    return fail(DIT_ERR_INVALID_ARG, "%s strides (%lld, %lld) must be multiples of %d elements, >= 0", name,
                (long long)row, (long long)head, unit);
  if ((rows > 1 && row < dh) || (heads > 1 && head < dh))
    return fail(DIT_ERR_INVALID_ARG, "%s strides (%lld, %lld): rows or heads of %d elements overlap", name,
                (long long)row, (long long)head, dh);
  if (row > (1 << 22) || head > (1L << 40))
    return fail(DIT_ERR_UNSUPPORTED, "%s strides (%lld, %lld) are too large", name, (long long)row, (long long)head);
  return DIT_OK;
}

// Whether two of o's dh-element pieces (row, head) share elements: dr rows and h heads
// apart they lie |dr row - h head| elements apart (or the sum, which is larger).
bool pieces_overlap(int64_t row, int64_t head, int64_t rows, int64_t heads, int64_t dh) {
  if (rows < 2 || heads < 2 || row >= (heads - 1) * head + dh || head >= (rows - 1) * row + dh) return false;
  for (int64_t h = 1; h < heads; ++h)
    for (int64_t dr = h * head / row; dr <= h * head / row + 1 && dr < rows; ++dr)
      if (dr * row - h * head < dh && h * head - dr * row < dh) return true;
  return false;
}

dit_status check_attn(const dit_attn_shape* s) {
  if (!s) return fail(DIT_ERR_INVALID_ARG, "shape is NULL");
  if (s->docs < 1 || s->heads < 1 || s->kv_heads < 1 || s->heads % s->kv_heads != 0)
    return fail(DIT_ERR_INVALID_ARG, "docs (%d) must be >= 1 and heads (%d) a multiple of kv_heads (%d)", s->docs,
                s->heads, s->kv_heads);
  if (s->docs > 65535 || s->heads > 65535) return fail(DIT_ERR_UNSUPPORTED, "more than 65535 documents or heads");
  if (s->head_dim != 64 && s->head_dim != 72 && s->head_dim != 128)
    return fail(DIT_ERR_UNSUPPORTED, "head_dim %d not supported (64, 72, 128)", s->head_dim);
  if (s->dtype != DIT_F32 && s->dtype != DIT_BF16) return fail(DIT_ERR_INVALID_ARG, "dtype %d unknown", s->dtype);
  if (s->mask < DIT_MASK_FULL || s->mask > DIT_MASK_PREFIX) return fail(DIT_ERR_INVALID_ARG, "mask %d unknown", s->mask);
  if (s->q_rows < 0 || s->k_rows < 0 || s->max_q < 0 || s->max_k < 0)
    return fail(DIT_ERR_INVALID_ARG, "q_rows (%d), k_rows (%d), max_q (%d), max_k (%d) must be >= 0", s->q_rows,
                s->k_rows, s->max_q, s->max_k);
  // (a grid has fewer than 2^32 threads: 16 for each query and head in fp32)
  if ((long)s->max_q * s->heads >= (s->dtype == DIT_BF16 ? 1L << 30 : 1L << 27) || (long)s->max_q * s->heads / s->kv_heads >= (1L << 24) ||
      s->max_k >= (1 << 30) || s->k_rows >= (1 << 30) || s->q_rows >= (1 << 30))
    return fail(DIT_ERR_UNSUPPORTED, "documents of %d queries and %d keys, or %d / %d rows, are too long", s->max_q,
                s->max_k, s->q_rows, s->k_rows);
  if (!(s->scale > 0.f) || !isfinite(s->scale) || !(s->cap >= 0.f) || !isfinite(s->cap))
    return fail(DIT_ERR_INVALID_ARG, "scale (%g) must be finite and > 0, cap (%g) finite and >= 0", s->scale, s->cap);
  // past these the scale times a score of 0 would be inf * 0, and the tanh's fp32
  // arithmetic (an error of cap * 2^-20 in a score) coarser than the probabilities
  if (s->scale > 0x1p100f || (s->cap > 0.f && (s->cap < 0x1p-20f || s->cap > 0x1p12f)))
    return fail(DIT_ERR_UNSUPPORTED, "scale (%g) > 2^100, or cap (%g) not 0 and not in 2^-20 .. 2^12", s->scale, s->cap);
  const int unit = s->dtype == DIT_BF16 ? 8 : 4, dh = s->head_dim;
  dit_status st;
  if ((st = check_strides("q", s->q_row, s->q_head, s->heads, s->q_rows, dh, unit)) != DIT_OK) return st;
  if ((st = check_strides("k", s->k_row, s->k_head, s->kv_heads, s->k_rows, dh, unit)) != DIT_OK) return st;
  if ((st = check_strides("v", s->v_row, s->v_head, s->kv_heads, s->k_rows, dh, unit)) != DIT_OK) return st;
  if ((st = check_strides("o", s->o_row, s->o_head, s->heads, s->q_rows, dh, unit)) != DIT_OK) return st;
  if (pieces_overlap(s->o_row, s->o_head, s->q_rows, s->heads, dh))
    return fail(DIT_ERR_INVALID_ARG, "o strides (%lld, %lld): rows and heads of %d elements overlap", (long long)s->o_row,
                (long long)s->o_head, dh);
  return DIT_OK;
}

DocAttnArgs attn_args(const dit_attn_shape* s) {
  DocAttnArgs a{};
  a.docs = s->docs;
  a.H = s->heads;
  a.Hk = s->kv_heads;
  a.G = s->heads / s->kv_heads;
  a.q_rows = s->q_rows;
  a.k_rows = s->k_rows;
  a.max_q = s->max_q < s->q_rows ? s->max_q : s->q_rows;
  a.max_k = s->max_k < s->k_rows ? s->max_k : s->k_rows;
  a.room_q = s->max_q;
  a.room_k = s->max_k;
  a.mask = s->mask;
  a.scale = s->scale;
  a.cap = s->cap;
  a.q_row = s->q_row;
  a.q_head = s->q_head;
  a.k_row = s->k_row;
  a.k_head = s->k_head;
  a.v_row = s->v_row;
  a.v_head = s->v_head;
  a.o_row = s->o_row;
  a.o_head = s->o_head;
  return a;
}

size_t attn_bytes(const dit_attn_shape* s, const DocAttnPlan& p) {
  return p.split > 1 ? (size_t)p.split * s->q_rows * s->heads * (s->head_dim + 4) * 4 : 0;
}

// ------------------------------------------------------------------ queries and keys
dit_status check_qk(const dit_qk_shape* s) {
  if (!s) return fail(DIT_ERR_INVALID_ARG, "shape is NULL");
  if (s->rows < 0 || s->heads < 0 || s->kv_heads < 0 || s->heads + (long)s->kv_heads < 1 || s->q_out_rows < 0 || s->k_out_rows < 0)
    return fail(DIT_ERR_INVALID_ARG, "rows (%d), heads (%d), kv_heads (%d), q_out_rows (%d), k_out_rows (%d) must be >= 0, one head at least",
                s->rows, s->heads, s->kv_heads, s->q_out_rows, s->k_out_rows);
  // (qk_segments() keeps a grid of so many rows below 2^32 threads)
  if (s->heads > 65535 || s->kv_heads > 65535 || s->rows > (1 << 24))
    return fail(DIT_ERR_UNSUPPORTED, "more than 65535 heads or 2^24 rows (%d)", s->rows);
  if (s->head_dim < 8 || s->head_dim % 8 != 0 || s->head_dim > 256)
    return fail(DIT_ERR_UNSUPPORTED, "head_dim %d not supported (multiples of 8 up to 256)", s->head_dim);
  if (s->dtype != DIT_F32 && s->dtype != DIT_BF16) return fail(DIT_ERR_INVALID_ARG, "dtype %d unknown", s->dtype);
  if (s->norm < DIT_NORM_NONE || s->norm > DIT_NORM_RMS) return fail(DIT_ERR_INVALID_ARG, "norm %d unknown", s->norm);
  if (s->pairing != DIT_PAIR_NEIGHBOURS && s->pairing != DIT_PAIR_HALVES)
    return fail(DIT_ERR_INVALID_ARG, "pairing %d unknown", s->pairing);
  if (s->norm != DIT_NORM_NONE && (!(s->eps >= 0x1p-126f) || !isfinite(s->eps)))
    return fail(DIT_ERR_INVALID_ARG, "eps (%g) must be finite and at least 2^-126", s->eps);
  if (s->axes < 0 || s->axes > 4) return fail(DIT_ERR_INVALID_ARG, "axes (%d) must be 0 .. 4", s->axes);
  long pairs = 0;
  for (int i = 0; i < s->axes; ++i) {
    if (s->pairs[i] < 0) return fail(DIT_ERR_INVALID_ARG, "pairs of axis %d (%d) must be >= 0", i, s->pairs[i]);
    pairs += s->pairs[i];
  }
  if (pairs * 2 > s->head_dim) return fail(DIT_ERR_INVALID_ARG, "%ld pairs do not fit head_dim (%d)", pairs, s->head_dim);
  if (s->pairing == DIT_PAIR_HALVES && pairs % 4 != 0)
    return fail(DIT_ERR_UNSUPPORTED, "%ld pairs of halves: not a multiple of 4", pairs);
  return DIT_OK;
}

// ------------------------------------------------------------------ linear
LinF4Plan plan_linear4(const dit_linear_shape* s) {
  return s->rows > 0 ? linear_fp4_plan(s->rows, s->out, s->in, s->dtype) : LinF4Plan{};
}

dit_status check_linear4(const dit_linear_shape* s) {
  if (!s) return fail(DIT_ERR_INVALID_ARG, "shape is NULL");
  if (s->rows < 0 || s->in < 32 || s->in % 32 != 0 || s->out < 1)
    return fail(DIT_ERR_INVALID_ARG, "rows (%d) must be >= 0, in (%d) a positive multiple of 32, out (%d) >= 1", s->rows,
                s->in, s->out);
  if (s->act != DIT_ACT_NONE && s->act != DIT_ACT_GELU) return fail(DIT_ERR_INVALID_ARG, "act %d unknown", s->act);
  if (s->dtype != DIT_F32 && s->dtype != DIT_BF16 && s->dtype != DIT_MXFP4)
    return fail(DIT_ERR_INVALID_ARG, "dtype %d is not DIT_F32, DIT_BF16 or DIT_MXFP4", s->dtype);
  if (s->dtype == DIT_MXFP4 && s->out % 32 != 0)
    return fail(DIT_ERR_INVALID_ARG, "out (%d) must be a multiple of 32 for a 4-bit output", s->out);
  if ((long)s->in > (1L << 22) || (long)s->out > (1L << 26) || (long)s->rows > (1L << 26) || plan_linear4(s).tile < 0)
    return fail(DIT_ERR_UNSUPPORTED, "product of %d x %d x %d is too large", s->rows, s->out, s->in);
  return DIT_OK;
}

LinF8Plan plan_linear(const dit_linear_shape* s) {
  return s->rows > 0 ? linear_fp8_plan(s->rows, s->out, s->in, s->dtype) : LinF8Plan{};
}

dit_status check_linear(const dit_linear_shape* s) {
  if (!s) return fail(DIT_ERR_INVALID_ARG, "shape is NULL");
  if (s->rows < 0 || s->in < 16 || s->in % 16 != 0 || s->out < 1)
    return fail(DIT_ERR_INVALID_ARG, "rows (%d) must be >= 0, in (%d) a positive multiple of 16, out (%d) >= 1", s->rows,
                s->in, s->out);
  if (s->act != DIT_ACT_NONE && s->act != DIT_ACT_GELU) return fail(DIT_ERR_INVALID_ARG, "act %d unknown", s->act);
  if (s->dtype != DIT_F32 && s->dtype != DIT_BF16 && s->dtype != DIT_E4M3)
    return fail(DIT_ERR_INVALID_ARG, "dtype %d unknown", s->dtype);
  // 32-bit lane offsets of a tile's rows, tile counts of one grid dimension
  if ((long)s->in > (1L << 22) || (long)s->out > (1L << 26) || (long)s->rows > (1L << 26) ||
      (((long)s->rows + 31) / 32) * (((long)s->out + 31) / 32) >= (1L << 31) || plan_linear(s).tile < 0)
    return fail(DIT_ERR_UNSUPPORTED, "product of %d x %d x %d is too large", s->rows, s->out, s->in);
  return DIT_OK;
}

dit_status check_ws(const void* ws, size_t bytes, size_t need) {
  if (need == 0) return DIT_OK;
  if (!ws || !aligned(ws, 256)) return fail(DIT_ERR_INVALID_ARG, "workspace NULL or not 256-byte aligned");
  if (bytes < need) return fail(DIT_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", bytes, need);
  return DIT_OK;
}

dit_status check_ptr(const void* p, const char* name, size_t align, bool optional) {
  if (!p && optional) return DIT_OK;
  if (!p || !aligned(p, align)) return fail(DIT_ERR_INVALID_ARG, "%s NULL or not %zu-byte aligned", name, align);
  return DIT_OK;
}

}  // namespace

#define TRY(expr)                        \
  do {                                   \
    const dit_status st_ = (expr);       \
    if (st_ != DIT_OK) return st_;       \
  } while (0)

size_t dit_attention_workspace_bytes(const dit_attn_shape* s) {
  if (check_attn(s) != DIT_OK) return BAD_SIZE;
  const DocAttnArgs a = attn_args(s);
  return attn_bytes(s, doc_attn_plan(a, s->head_dim, s->dtype));
}

dit_status dit_attention(const dit_attn_shape* s, const void* q, const void* k, const void* v, void* o,
                         const int32_t* q_start, const int32_t* k_start, const int32_t* k_len, const int32_t* prefix,
                         const float* slopes, void* workspace, size_t ws_bytes, void* stream) {
  TRY(check_attn(s));
  if ((s->mask == DIT_MASK_PREFIX) != (prefix != nullptr))
    return fail(DIT_ERR_INVALID_ARG, "prefix is given with DIT_MASK_PREFIX and only then");
  if (!q_start && (long)s->docs * s->max_q > s->q_rows)
    return fail(DIT_ERR_INVALID_ARG, "%d rooms of %d query rows do not fit q_rows (%d)", s->docs, s->max_q, s->q_rows);
  if (!k_start && (long)s->docs * s->max_k > s->k_rows)
    return fail(DIT_ERR_INVALID_ARG, "%d rooms of %d keys do not fit k_rows (%d)", s->docs, s->max_k, s->k_rows);
  DocAttnArgs a = attn_args(s);
  TRY(check_ptr(q, "q", 16, s->q_rows == 0));
  TRY(check_ptr(k, "k", 16, s->k_rows == 0));
  TRY(check_ptr(v, "v", 16, s->k_rows == 0));
  TRY(check_ptr(o, "o", 16, s->q_rows == 0));
  TRY(check_ptr(q_start, "q_start", 4, true));
  TRY(check_ptr(k_start, "k_start", 4, true));
  TRY(check_ptr(k_len, "k_len", 4, true));
  TRY(check_ptr(prefix, "prefix", 4, true));
  TRY(check_ptr(slopes, "slopes", 4, true));
  const DocAttnPlan p = doc_attn_plan(a, s->head_dim, s->dtype);
  TRY(check_ws(workspace, ws_bytes, attn_bytes(s, p)));
  if (a.max_q == 0) return DIT_OK;
  a.q = q;
  a.k = k;
  a.v = v;
  a.o = o;
  a.q_start = q_start;
  a.k_start = k_start;
  a.k_len = k_len;
  a.prefix = prefix;
  a.slopes = slopes;
  a.split = p.split;
  a.part = (float*)workspace;
  const hipStream_t st = (hipStream_t)stream;
  const double e = s->dtype == DIT_BF16 ? 2 : 4;
  // the documents' lengths live on the device: what the rows could need at most
  const double flops = 4.0 * s->head_dim * s->heads * (double)s->q_rows * a.max_k;
  const double bytes = 2 * e * s->head_dim * ((double)s->heads * s->q_rows + (double)s->kv_heads * s->k_rows);
  HIP_TRY(timed(DIT_K_ATTENTION, flops, bytes, st, [&]() {
    hipError_t r = s->dtype == DIT_BF16 ? launch_doc_attn_bf16(a, p, s->head_dim, st)
                                        : launch_doc_attn_f32(a, p, s->head_dim, st);
    if (r == hipSuccess && p.split > 1) r = launch_doc_attn_merge(a, s->head_dim, s->dtype, st);
    return r;
  }));
  return DIT_OK;
}

dit_status dit_quantize_fp8(int32_t rows, int32_t cols, int32_t block_rows, int32_t dtype, const void* x,
                            int64_t x_row, void* codes, float* scale, void* stream) {
  if (rows < 0 || cols < 8 || cols % 8 != 0 || x_row % 8 != 0 || x_row < cols)
    return fail(DIT_ERR_INVALID_ARG, "rows (%d) must be >= 0, cols (%d) and x_row (%lld) multiples of 8, x_row >= cols",
                rows, cols, (long long)x_row);
  if (block_rows != 1 && block_rows != 128) return fail(DIT_ERR_INVALID_ARG, "block_rows (%d) must be 1 or 128", block_rows);
  if (dtype != DIT_F32 && dtype != DIT_BF16) return fail(DIT_ERR_INVALID_ARG, "dtype %d unknown", dtype);
  // (a grid has fewer than 2^32 threads: 16 for a block of one row, 256 for one of 128 rows)
  const long blocks = (long)rows * (((long)cols + 127) / 128);
  if (x_row > (1L << 40) || cols > (1 << 30) || (block_rows == 1 ? blocks >= (1L << 28) - 16 : rows > 65535 * 128))
    return fail(DIT_ERR_UNSUPPORTED, "%d rows of %d columns are too many", rows, cols);
  if (rows == 0) return DIT_OK;
  TRY(check_ptr(x, "x", 16, false));
  TRY(check_ptr(codes, "codes", 16, false));
  TRY(check_ptr(scale, "scale", 4, false));
  const hipStream_t st = (hipStream_t)stream;
  const double n = (double)rows * cols;
  HIP_TRY(timed(DIT_K_OTHER, 3 * n, n * (dtype == DIT_BF16 ? 3 : 5), st, [&]() {
    return launch_quantize_fp8(rows, cols, block_rows, dtype, x, x_row, codes, scale, st);
  }));
  return DIT_OK;
}

size_t dit_linear_fp8_workspace_bytes(const dit_linear_shape* s) {
  if (check_linear(s) != DIT_OK) return BAD_SIZE;
  return plan_linear(s).bytes;
}

dit_status dit_linear_fp8(const dit_linear_shape* s, const void* a, const float* a_scale, const void* w,
                          const float* w_scale, const void* bias, void* out, float* out_scale, void* workspace,
                          size_t ws_bytes, void* stream) {
  TRY(check_linear(s));
  if (s->dtype != DIT_E4M3 && out_scale) return fail(DIT_ERR_INVALID_ARG, "out_scale is for 8-bit outputs");
  if (s->rows == 0) return DIT_OK;
  TRY(check_ptr(a, "a", 16, false));
  TRY(check_ptr(w, "w", 16, false));
  TRY(check_ptr(a_scale, "a_scale", 4, false));
  TRY(check_ptr(w_scale, "w_scale", 4, false));
  TRY(check_ptr(bias, "bias", 16, true));
  TRY(check_ptr(out, "out", 16, false));
  TRY(check_ptr(out_scale, "out_scale", 4, s->dtype != DIT_E4M3));
  const LinF8Plan p = plan_linear(s);
  TRY(check_ws(workspace, ws_bytes, p.bytes));
  LinF8Args l{};
  l.a = (const uint8_t*)a;
  l.w = (const uint8_t*)w;
  l.a_scale = a_scale;
  l.w_scale = w_scale;
  l.bias = bias;
  l.out = out;
  l.out_scale = out_scale;
  l.M = s->rows;
  l.N = s->out;
  l.K = s->in;
  l.act = s->act;
  l.dtype = s->dtype;
  l.n_full = p.n_full;
  l.split = p.split;
  l.part = (float*)workspace;
  const hipStream_t st = (hipStream_t)stream;
  const double M = l.M, N = l.N, K = l.K;
  HIP_TRY(timed(DIT_K_OTHER, 2 * M * N * K, M * K + N * K + M * N * (l.dtype == 0 ? 4 : l.dtype == 1 ? 2 : 1), st,
                [&]() { return launch_linear_fp8(l, p.tile, st); }));
  return DIT_OK;
}

dit_status dit_norm_residual(const dit_norm_shape* s, const float* x, float* x_out, const void* y, const float* w_post,
                             const float* gate, const float* w_pre, const float* shift, const float* scale,
                             const int32_t* row_batch, void* h, float* h_scale, void* stream) {
  if (!s) return fail(DIT_ERR_INVALID_ARG, "shape is NULL");
  if (s->rows < 0 || s->hidden < 8 || s->hidden % 8 != 0 || s->batch < 1)
    return fail(DIT_ERR_INVALID_ARG, "rows (%d) must be >= 0, hidden (%d) a positive multiple of 8, batch (%d) >= 1",
                s->rows, s->hidden, s->batch);
  // (a grid has fewer than 2^32 threads: 64 for a row, 256 from 4097 columns on)
  if (s->hidden > 8192 || s->rows > (s->hidden > 4096 ? (1 << 24) - 1 : 1 << 25))
    return fail(DIT_ERR_UNSUPPORTED, "%d rows of %d: at most 8192 columns, and 2^25 rows (2^24 - 1 of more than 4096)",
                s->rows, s->hidden);
  if (s->post < DIT_NORM_NONE || s->post > DIT_NORM_RMS || s->pre < DIT_NORM_LAYER || s->pre > DIT_NORM_RMS)
    return fail(DIT_ERR_INVALID_ARG, "norms (post %d, pre %d) unknown", s->post, s->pre);
  if ((s->y_dtype != DIT_F32 && s->y_dtype != DIT_BF16) || s->h_dtype < DIT_F32 || s->h_dtype > DIT_E4M3)
    return fail(DIT_ERR_INVALID_ARG, "y_dtype %d or h_dtype %d unknown", s->y_dtype, s->h_dtype);
  if (!(s->eps > 0.f) || !isfinite(s->eps) || !isfinite(s->res_scale))
    return fail(DIT_ERR_INVALID_ARG, "eps (%g) must be finite and > 0, res_scale (%g) finite", s->eps, s->res_scale);
  if ((gate || shift || scale) && (s->mod_stride % 4 != 0 || s->mod_stride < 0 ||
                                   (s->batch > 1 && s->mod_stride < s->hidden) || s->mod_stride > (1L << 40)))
    return fail(DIT_ERR_INVALID_ARG, "mod_stride (%lld) must be a multiple of 4 and at least hidden",
                (long long)s->mod_stride);
  if (!y && (gate || w_post || s->post != DIT_NORM_NONE))
    return fail(DIT_ERR_INVALID_ARG, "post, w_post and gate need y");
  if (y && s->post == DIT_NORM_NONE && w_post) return fail(DIT_ERR_INVALID_ARG, "w_post needs a post norm");
  if ((shift != nullptr) != (scale != nullptr)) return fail(DIT_ERR_INVALID_ARG, "shift and scale come together");
  if (!h && (w_pre || shift || h_scale)) return fail(DIT_ERR_INVALID_ARG, "w_pre, shift, scale and h_scale need h");
  if (!h && !x_out) return fail(DIT_ERR_INVALID_ARG, "neither x_out nor h is given");
  if (y && !x_out) return fail(DIT_ERR_INVALID_ARG, "y needs x_out");
  if (h && (s->h_dtype == DIT_E4M3) != (h_scale != nullptr))
    return fail(DIT_ERR_INVALID_ARG, "h_scale is given with an 8-bit h and only then");
  if (s->rows == 0) return DIT_OK;
  TRY(check_ptr(x, "x", 16, false));
  TRY(check_ptr(x_out, "x_out", 16, true));
  TRY(check_ptr(y, "y", 16, true));
  TRY(check_ptr(w_post, "w_post", 16, true));
  TRY(check_ptr(gate, "gate", 16, true));
  TRY(check_ptr(w_pre, "w_pre", 16, true));
  TRY(check_ptr(shift, "shift", 16, true));
  TRY(check_ptr(scale, "scale", 16, true));
  TRY(check_ptr(row_batch, "row_batch", 4, true));
  TRY(check_ptr(h, "h", 16, true));
  TRY(check_ptr(h_scale, "h_scale", 4, true));
  NormResArgs a{};
  a.x = x;
  a.x_out = x_out;
  a.y = y;
  a.w_post = w_post;
  a.gate = gate;
  a.w_pre = w_pre;
  a.shift = shift;
  a.scale = scale;
  a.row_batch = row_batch;
  a.h = h;
  a.h_scale = h_scale;
  a.rows = s->rows;
  a.D = s->hidden;
  a.batch = s->batch;
  a.per_batch = (int)(((long)s->rows + s->batch - 1) / s->batch);
  a.post = s->post;
  a.pre = s->pre;
  a.y_dtype = s->y_dtype;
  a.h_dtype = s->h_dtype;
  a.eps = s->eps;
  a.res_scale = s->res_scale;
  a.mod_stride = (long)s->mod_stride;
  const hipStream_t st = (hipStream_t)stream;
  const double n = (double)s->rows * s->hidden;
  const double bytes = n * (4 + (x_out ? 4 : 0) + (y ? (s->y_dtype == DIT_BF16 ? 2 : 4) : 0) +
                            (h ? (s->h_dtype == DIT_F32 ? 4 : s->h_dtype == DIT_BF16 ? 2 : 1) : 0));
  HIP_TRY(timed(DIT_K_LN_MOD, 16 * n, bytes, st, [&]() { return launch_norm_residual(a, st); }));
  return DIT_OK;
}

// rows [rows, cols] of quantised blocks of 32, and of the values x they stand for
static dit_status check_blocks(int32_t rows, int32_t cols, int32_t dtype, int64_t x_row) {
  if (rows < 0 || cols < 32 || cols % 32 != 0 || x_row % 8 != 0 || x_row < cols)
    return fail(DIT_ERR_INVALID_ARG, "rows (%d) must be >= 0, cols (%d) a positive multiple of 32, x_row (%lld) one of 8 and >= cols",
                rows, cols, (long long)x_row);
  if (dtype != DIT_F32 && dtype != DIT_BF16) return fail(DIT_ERR_INVALID_ARG, "dtype %d unknown", dtype);
  // (a grid has fewer than 2^32 threads: 256 for 8 rows of 256 columns)
  if (x_row > (1L << 40) || cols > (1 << 30) || (((long)rows + 7) / 8) * (((long)cols + 255) / 256) >= (1L << 24))
    return fail(DIT_ERR_UNSUPPORTED, "%d rows of %d columns are too many", rows, cols);
  return DIT_OK;
}

dit_status dit_quantize_fp4(int32_t rows, int32_t cols, int32_t dtype, const void* x, int64_t x_row, void* codes, void* scale,
                            void* stream) {
  TRY(check_blocks(rows, cols, dtype, x_row));
  if (rows == 0) return DIT_OK;
  TRY(check_ptr(x, "x", 16, false));
  TRY(check_ptr(codes, "codes", 16, false));
  TRY(check_ptr(scale, "scale", 16, false));
  const hipStream_t st = (hipStream_t)stream;
  const double n = (double)rows * cols;
  HIP_TRY(timed(DIT_K_OTHER, 3 * n, n * ((dtype == DIT_BF16 ? 2 : 4) + 0.53125), st, [&]() {
    return launch_quantize_fp4(rows, cols, dtype, x, x_row, codes, scale, st);
  }));
  return DIT_OK;
}

dit_status dit_dequantize_fp4(int32_t rows, int32_t cols, int32_t dtype, const void* codes, const void* scale, void* x,
                              int64_t x_row, void* stream) {
  TRY(check_blocks(rows, cols, dtype, x_row));
  if (rows == 0) return DIT_OK;
  TRY(check_ptr(codes, "codes", 16, false));
  TRY(check_ptr(scale, "scale", 16, false));
  TRY(check_ptr(x, "x", 16, false));
  const hipStream_t st = (hipStream_t)stream;
  const double n = (double)rows * cols;
  HIP_TRY(timed(DIT_K_OTHER, n, n * ((dtype == DIT_BF16 ? 2 : 4) + 0.53125), st, [&]() {
    return launch_dequantize_fp4(rows, cols, dtype, codes, scale, x, x_row, st);
  }));
  return DIT_OK;
}

size_t dit_linear_fp4_workspace_bytes(const dit_linear_shape* s) {
  if (check_linear4(s) != DIT_OK) return BAD_SIZE;
  return plan_linear4(s).bytes;
}

dit_status dit_linear_fp4(const dit_linear_shape* s, const void* a, const void* a_scale, const void* w, const void* w_scale,
                          const void* bias, void* out, void* out_scale, void* workspace, size_t ws_bytes, void* stream) {
  TRY(check_linear4(s));
  if (s->dtype != DIT_MXFP4 && out_scale) return fail(DIT_ERR_INVALID_ARG, "out_scale is for 4-bit outputs");
  if (s->rows == 0) return DIT_OK;
  TRY(check_ptr(a, "a", 16, false));
  TRY(check_ptr(w, "w", 16, false));
  TRY(check_ptr(a_scale, "a_scale", 16, false));
  TRY(check_ptr(w_scale, "w_scale", 16, false));
  TRY(check_ptr(bias, "bias", 16, true));
  TRY(check_ptr(out, "out", 16, false));
  TRY(check_ptr(out_scale, "out_scale", 16, s->dtype != DIT_MXFP4));
  const LinF4Plan p = plan_linear4(s);
  TRY(check_ws(workspace, ws_bytes, p.bytes));
  LinF4Args l{};
  l.a = (const uint8_t*)a;
  l.w = (const uint8_t*)w;
  l.a_scale = (const uint8_t*)a_scale;
  l.w_scale = (const uint8_t*)w_scale;
  l.bias = bias;
  l.out = out;
  l.out_scale = (uint8_t*)out_scale;
  l.M = s->rows;
  l.N = s->out;
  l.K = s->in;
  l.act = s->act;
  l.dtype = s->dtype;
  l.split = p.split;
  l.part = (float*)workspace;
  const hipStream_t st = (hipStream_t)stream;
  const double M = l.M, N = l.N, K = l.K, e = l.dtype == DIT_F32 ? 4 : l.dtype == DIT_BF16 ? 2 : 0.53125;
  HIP_TRY(timed(DIT_K_OTHER, 2 * M * N * K, 0.53125 * K * (M + N) + M * N * e, st, [&]() { return launch_linear_fp4(l, p, st); }));
  return DIT_OK;
}

dit_status dit_qk_norm_rope(const dit_qk_shape* s, const void* q, const void* k, const void* v, void* q_out, void* k_out,
                            void* v_out, const float* w_q, const float* w_k, const int32_t* pos, const double* freqs,
                            const int32_t* q_dst, const int32_t* k_dst, void* stream) {
  TRY(check_qk(s));
  const int unit = s->dtype == DIT_BF16 ? 8 : 4, dh = s->head_dim, R = s->rows, H = s->heads, Hk = s->kv_heads;
  // (tensors without rows may come as NULL)
  if ((v != nullptr) != (v_out != nullptr) && R != 0 && !(v && s->k_out_rows == 0))
    return fail(DIT_ERR_INVALID_ARG, "v and v_out come together");
  if (v && !v_out) v = nullptr;  // none of its rows has a place
  if (v && Hk == 0) return fail(DIT_ERR_INVALID_ARG, "v has kv_heads heads, which are none");
  if (s->norm == DIT_NORM_NONE && (w_q || w_k)) return fail(DIT_ERR_INVALID_ARG, "w_q and w_k need a norm");
  struct {
    const char* name;
    int64_t row, head;
    int heads, rows;
    bool out;
  } const t[6] = {{"q", s->q_row, s->q_head, H, R, false},
                  {"k", s->k_row, s->k_head, Hk, R, false},
                  {"v", s->v_row, s->v_head, v ? Hk : 0, R, false},
                  {"q_out", s->q_out_row, s->q_out_head, H, s->q_out_rows, true},
                  {"k_out", s->k_out_row, s->k_out_head, Hk, s->k_out_rows, true},
                  {"v_out", s->v_out_row, s->v_out_head, v ? Hk : 0, s->k_out_rows, true}};
  for (const auto& x : t) {
    if (x.heads == 0) continue;
    TRY(check_strides(x.name, x.row, x.head, x.heads, x.rows, dh, unit));
    if (x.out && pieces_overlap(x.row, x.head, x.rows, x.heads, dh))
      return fail(DIT_ERR_INVALID_ARG, "%s strides (%lld, %lld): rows and heads of %d elements overlap", x.name, (long long)x.row,
                  (long long)x.head, dh);
  }
  if (H && !q_dst && s->q_out_rows < R)
    return fail(DIT_ERR_INVALID_ARG, "q_out_rows (%d): %d rows do not fit without q_dst", s->q_out_rows, R);
  if (Hk && !k_dst && s->k_out_rows < R)
    return fail(DIT_ERR_INVALID_ARG, "k_out_rows (%d): %d rows do not fit without k_dst", s->k_out_rows, R);
  // in place: every head is read and written by the same lanes, where it stays at its place
  if ((H && q && q == q_out && (q_dst || s->q_row != s->q_out_row || s->q_head != s->q_out_head)) ||
      (Hk && k && k == k_out && (k_dst || s->k_row != s->k_out_row || s->k_head != s->k_out_head)) ||
      (v && v == v_out && (k_dst || s->v_row != s->v_out_row || s->v_head != s->v_out_head)))
    return fail(DIT_ERR_INVALID_ARG, "in place only with the same strides and without q_dst or k_dst");
  if (R == 0) return DIT_OK;
  int pairs = 0, ends[4] = {};
  for (int i = 0; i < 4; ++i) ends[i] = pairs += i < s->axes ? s->pairs[i] : 0;
  TRY(check_ptr(q, "q", 16, H == 0));
  TRY(check_ptr(k, "k", 16, Hk == 0));
  TRY(check_ptr(v, "v", 16, true));
  TRY(check_ptr(q_out, "q_out", 16, H == 0 || s->q_out_rows == 0));
  TRY(check_ptr(k_out, "k_out", 16, Hk == 0 || s->k_out_rows == 0));
  TRY(check_ptr(v_out, "v_out", 16, true));
  TRY(check_ptr(w_q, "w_q", 16, true));
  TRY(check_ptr(w_k, "w_k", 16, true));
  TRY(check_ptr(pos, "pos", 4, pairs == 0));
  TRY(check_ptr(freqs, "freqs", 8, pairs == 0));
  TRY(check_ptr(q_dst, "q_dst", 4, true));
  TRY(check_ptr(k_dst, "k_dst", 4, true));
  QkArgs a{};
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_out = q_out;
  a.k_out = k_out;
  a.v_out = v_out;
  a.w_q = w_q;
  a.w_k = w_k;
  a.pos = pos;
  a.freqs = freqs;
  a.q_dst = q_dst;
  a.k_dst = k_dst;
  a.rows = R;
  a.H = H;
  a.Hk = Hk;
  a.Hv = v ? Hk : 0;
  a.dh = dh;
  a.norm = s->norm;
  a.halves = s->pairing == DIT_PAIR_HALVES;
  a.axes = s->axes;
  a.P = pairs;
  for (int i = 0; i < 3; ++i) a.axis_end[i] = ends[i];
  a.q_out_rows = s->q_out_rows;
  a.k_out_rows = s->k_out_rows;
  a.eps = s->eps;
  a.q_row = s->q_row;
  a.q_head = s->q_head;
  a.k_row = s->k_row;
  a.k_head = s->k_head;
  a.v_row = s->v_row;
  a.v_head = s->v_head;
  a.qo_row = s->q_out_row;
  a.qo_head = s->q_out_head;
  a.ko_row = s->k_out_row;
  a.ko_head = s->k_out_head;
  a.vo_row = s->v_out_row;
  a.vo_head = s->v_out_head;
  const hipStream_t st = (hipStream_t)stream;
  const double n = (double)R * dh;
  HIP_TRY(timed(DIT_K_OTHER, 8 * n * (H + Hk), 2 * n * (H + Hk + a.Hv) * (s->dtype == DIT_BF16 ? 2 : 4), st,
                [&]() { return launch_qk_norm_rope(a, s->dtype, st); }));
  return DIT_OK;
}
