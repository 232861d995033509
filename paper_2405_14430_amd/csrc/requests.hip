// C entry points of the operators on packed rows: checks of arguments, then one call into the launch functions.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include <algorithm>

#include "mx.h"
#include "requests.h"

using namespace pf;

namespace {

constexpr int64_t kMaxKeys = (1ll << 31) - 4096;   // of a sequence: the kernels round key numbers up to whole tiles of chunks in 32 bits
constexpr int kMaxRows = 1 << 24;   // rows of one call of the row-wise operators
constexpr int kMaxSeqs = 1 << 30;   // wave_search probes up to 64 places behind the last one, in 32 bits

bool dt_ok(int dt) { return dt == PF_F32 || dt == PF_BF16; }
bool aligned(const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
bool row_stride_ok(int64_t ld, int64_t width, int dt) { return ld >= width && ld % (16 / (int64_t)dt_size(dt)) == 0; }
bool head_ok(int dh) { return dh >= 8 && dh <= 128 && dh % 8 == 0; }

pf_status refuse(pf_status st, const char *fmt, ...) {
  char text[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(text, sizeof(text), fmt, ap);
  va_end(ap);
  return note_error(st, text);
}
pf_status launched(hipError_t e, const char *what) {
  return e == hipSuccess ? PF_OK : refuse(PF_ERR_DEVICE, "%s: %s", what, hipGetErrorString(e));
}

// nullptr, or what is wrong with a rotation for heads of head_dim channels
const char *rope_wrong(const pf_rope &r, int head_dim) {
  if (r.layout != PF_ROPE_INTERLEAVED && r.layout != PF_ROPE_HALF) return "rope: unknown layout";
  if (r.n_axes < 1 || r.n_axes > PF_ROPE_MAX_AXES) return "rope: 1 to 3 axes";
  int sum = 0;
  for (int i = 0; i < r.n_axes; ++i) {
    if (r.axis_dim[i] < 2 || r.axis_dim[i] % 2 || r.axis_dim[i] > 2 * PF_ROPE_MAX_PAIRS) return "rope: axis_dim must be even, 2 .. 128";
    sum += r.axis_dim[i];
  }
  if (sum > head_dim) return "rope: the axes are wider than the head";
  if (!(r.magnitude > 0.f) || !isfinite(r.magnitude)) return "rope: magnitude must be positive and finite";
  return nullptr;
}

// what pf_kv_pages and pf_kv_mx_pages have in common
template <typename P>
pf_status page_sizes_check(const P *p, const char *who) {
  if (!head_ok(p->head_dim) || p->kv_heads < 1 || p->kv_heads > 65536 || p->n_seqs < 0 || p->n_seqs > kMaxSeqs || p->max_pages < 1 || p->n_pages < 1)
    return refuse(PF_ERR_SHAPE, "%s: pages: head_dim %d, kv_heads %d, n_seqs %d, max_pages %d, n_pages %d", who, p->head_dim, p->kv_heads,
                  p->n_seqs, p->max_pages, p->n_pages);
  if (p->page_size < 16 || p->page_size > 1024 || (p->page_size & (p->page_size - 1)))
    return refuse(PF_ERR_SHAPE, "%s: page_size %d is no power of two in 16 .. 1024", who, p->page_size);
  return PF_OK;
}

pf_status pages_check(int dtype, const pf_kv_pages *p, const char *who) {
  if (!p->k || !p->v || !p->table) return refuse(PF_ERR_NULL, "%s: k, v or table of the pages is NULL", who);
  if (pf_status st = page_sizes_check(p, who); st != PF_OK) return st;
  const int64_t block = (int64_t)p->kv_heads * p->page_size * p->head_dim;
  if (!row_stride_ok(p->k_page_stride, block, dtype) || !row_stride_ok(p->v_page_stride, block, dtype) || !aligned(p->k, 16) || !aligned(p->v, 16))
    return refuse(PF_ERR_SHAPE, "%s: pages: strides of at least %lld elements in whole 16 bytes, pointers 16-byte aligned", who, (long long)block);
  if (p->k_page_stride > INT64_MAX / 8 / p->n_pages || p->v_page_stride > INT64_MAX / 8 / p->n_pages)
    return refuse(PF_ERR_SHAPE, "%s: pages: n_pages * stride overflows", who);
  return PF_OK;
}

pf_status mx_pages_check(const pf_kv_mx_pages *p, const char *who) {
  if (!p->k || !p->v || !p->k_scale || !p->v_scale || !p->table) return refuse(PF_ERR_NULL, "%s: k, v, their scales or table of the pages is NULL", who);
  if (p->format != PF_MX_E4M3 && p->format != PF_MX_E2M1) return refuse(PF_ERR_DTYPE, "%s: pages: format %d", who, p->format);
  if (pf_status st = page_sizes_check(p, who); st != PF_OK) return st;
  const int64_t rows = (int64_t)p->kv_heads * p->page_size, block = rows * mx_row_bytes(p->format, p->head_dim), scales = rows * mx_blocks(p->head_dim);
  if (p->k_page_stride < block || p->v_page_stride < block || p->k_page_stride % 16 || p->v_page_stride % 16 || !aligned(p->k, 16) || !aligned(p->v, 16))
    return refuse(PF_ERR_SHAPE, "%s: pages: strides of at least %lld bytes in whole 16, pointers 16-byte aligned", who, (long long)block);
  if (p->k_scale_stride < scales || p->v_scale_stride < scales)
    return refuse(PF_ERR_SHAPE, "%s: pages: strides of at least %lld bytes between the scales of pages", who, (long long)scales);
  const int64_t most = std::max(std::max(p->k_page_stride, p->v_page_stride), std::max(p->k_scale_stride, p->v_scale_stride));
  if (most > INT64_MAX / 8 / p->n_pages) return refuse(PF_ERR_SHAPE, "%s: pages: n_pages * stride overflows", who);
  return PF_OK;
}
Pages mx_places(const pf_kv_mx_pages &p) {
  return Pages{p.k, p.v, p.k_page_stride, p.v_page_stride, p.table, p.n_pages, __builtin_ctz((unsigned)p.page_size), p.max_pages};
}
MxPages mx_numbers(const pf_kv_mx_pages &p) {
  return MxPages{p.format, mx_row_bytes(p.format, p.head_dim), mx_blocks(p.head_dim), (uint8_t *)p.k_scale, (uint8_t *)p.v_scale, p.k_scale_stride, p.v_scale_stride};
}

// The norm of a side's heads into `to`, or what is wrong with it.
pf_status head_norm(const pf_norm *n, NormSide &to, const char *who) {
  to = NormSide{PF_NORM_NONE, 0.f, nullptr, nullptr};
  if (!n) return PF_OK;
  if (n->kind < PF_NORM_NONE || n->kind > PF_NORM_LAYER) return refuse(PF_ERR_CONFIG, "%s: norm kind %d", who, n->kind);
  if (n->kind != PF_NORM_NONE && !(n->eps >= 0.f)) return refuse(PF_ERR_CONFIG, "%s: norm eps", who);
  if (n->kind == PF_NORM_NONE && (n->weight || n->bias)) return refuse(PF_ERR_CONFIG, "%s: weights of a norm of kind NONE", who);
  if (!aligned(n->weight, 16) || !aligned(n->bias, 16)) return refuse(PF_ERR_SHAPE, "%s: alignment of norm weights", who);
  to = NormSide{n->kind, n->eps, n->weight, n->bias};
  return PF_OK;
}

// a launch's query rows and heads: rows * heads is counted in 32 bits in the kernels
bool heads_ok(int total_q, int n_heads, int kv_heads) {
  return n_heads >= 1 && kv_heads >= 1 && kv_heads <= 65536 && n_heads % kv_heads == 0 && (int64_t)total_q * n_heads < (1ll << 31) - 4096;
}

}  // namespace

extern "C" {

pf_status pf_rope_init(const pf_rope_config *c, pf_rope *out) {
  if (!c || !out) return refuse(PF_ERR_NULL, "pf_rope_init: NULL");
  pf_rope r{};
  r.layout = c->layout;
  r.n_axes = c->n_axes;
  r.magnitude = c->magnitude;
  for (int i = 0; i < PF_ROPE_MAX_AXES; ++i) r.axis_dim[i] = i < c->n_axes ? c->axis_dim[i] : 0;
  if (const char *w = rope_wrong(r, 2 * PF_ROPE_MAX_PAIRS)) return refuse(PF_ERR_CONFIG, "%s", w);
  if (!(c->theta > 1.f) || !isfinite(c->theta)) return refuse(PF_ERR_CONFIG, "rope: theta must be > 1 and finite");
  if (c->scaling < PF_ROPE_SCALE_NONE || c->scaling > PF_ROPE_SCALE_RAMP_INDEX) return refuse(PF_ERR_CONFIG, "rope: unknown scaling");
  if (c->scaling != PF_ROPE_SCALE_NONE && (!(c->factor >= 1.f) || !isfinite(c->factor))) return refuse(PF_ERR_CONFIG, "rope: factor must be >= 1 and finite");
  if (c->scaling >= PF_ROPE_SCALE_RAMP_TURNS && (!(c->low > 0.f) || !(c->high > c->low) || !isfinite(c->high) || c->original_len < 1))
    return refuse(PF_ERR_CONFIG, "rope: a ramp needs high > low > 0 and original_len >= 1");
  const double two_pi = 6.283185307179586476925, factor = c->factor, len = c->original_len;
  int at = 0;
  for (int a = 0; a < r.n_axes; ++a) {
    const int w = r.axis_dim[a];
    const double theta = c->scaling == PF_ROPE_SCALE_NTK && w > 2 ? c->theta * pow(factor, (double)w / (w - 2)) : (double)c->theta;
    double from = 0, to = 0;   // RAMP_INDEX: the ramp's ends as pair indexes
    if (c->scaling == PF_ROPE_SCALE_RAMP_INDEX) {
      from = floor(w * log(len / (two_pi * c->high)) / (2 * log(theta)));
      to = ceil(w * log(len / (two_pi * c->low)) / (2 * log(theta)));
      from = from > 0 ? from : 0;
      to = to < w - 1 ? to : w - 1;
    }
    for (int i = 0; i < w / 2; ++i) {
      const double f = pow(theta, -2.0 * i / w) / two_pi;   // turns per position
      double keep = 1;                                      // share of the unchanged frequency
      if (c->scaling == PF_ROPE_SCALE_LINEAR) keep = 0;
      if (c->scaling == PF_ROPE_SCALE_RAMP_TURNS) keep = (len * f - c->low) / ((double)c->high - c->low);
      if (c->scaling == PF_ROPE_SCALE_RAMP_INDEX) keep = 1 - (i - from) / (to - from > 1e-3 ? to - from : 1e-3);
      keep = keep < 0 ? 0 : keep > 1 ? 1 : keep;
      r.turns[at++] = c->scaling == PF_ROPE_SCALE_NONE || c->scaling == PF_ROPE_SCALE_NTK ? f : f * keep + f / factor * (1 - keep);
    }
  }
  *out = r;
  return PF_OK;
}

pf_status pf_op_rope(int dtype, const pf_rope *rope, const int32_t *pos, const void *x, int64_t ldx, void *out, int64_t ldo,
                     int tokens, int n_heads, int head_dim, void *stream) {
  if (tokens < 0) return refuse(PF_ERR_SHAPE, "pf_op_rope: %d tokens", tokens);
  if (!dt_ok(dtype)) return refuse(PF_ERR_DTYPE, "pf_op_rope: dtype %d", dtype);
  if (tokens == 0) return PF_OK;
  if (!rope || !pos || !x || !out) return refuse(PF_ERR_NULL, "pf_op_rope: NULL");
  if (!head_ok(head_dim) || n_heads < 1 || n_heads > 65536) return refuse(PF_ERR_SHAPE, "pf_op_rope: %d heads of %d", n_heads, head_dim);
  const int64_t d = (int64_t)n_heads * head_dim;
  if (!row_stride_ok(ldx, d, dtype) || !row_stride_ok(ldo, d, dtype) || !aligned(x, 16) || !aligned(out, 16) || !aligned(pos, 4))
    return refuse(PF_ERR_SHAPE, "pf_op_rope: row strides %lld, %lld for rows of %lld, or alignment", (long long)ldx, (long long)ldo, (long long)d);
  if (tokens > kMaxRows) return refuse(PF_ERR_SHAPE, "pf_op_rope: %d tokens are more than %d", tokens, kMaxRows);
  if (x == out && ldx != ldo) return refuse(PF_ERR_SHAPE, "pf_op_rope: in place with two row strides");
  if (const char *w = rope_wrong(*rope, head_dim)) return refuse(PF_ERR_CONFIG, "%s", w);
  RopeRows a{};
  a.dt = dtype; a.rope = rope; a.pos = pos; a.tokens = tokens; a.head_dim = head_dim;
  a.q = x; a.ldq = ldx; a.q_out = out; a.ldqo = ldo; a.n_heads = n_heads;
  return launched(launch_rope_rows(a, (hipStream_t)stream), "pf_op_rope");
}

pf_status pf_op_kv_append(int dtype, const pf_kv_pages *pages, const void *k, int64_t ldk, const void *v, int64_t ldv,
                          const int32_t *cu, const int32_t *first, int tokens, const pf_rope *rope, const int32_t *pos,
                          const void *q, int64_t ldq, void *q_out, int64_t ldqo, int n_heads, void *stream) {
  if (tokens < 0 || n_heads < 0 || n_heads > 65536) return refuse(PF_ERR_SHAPE, "pf_op_kv_append: %d tokens, %d heads", tokens, n_heads);
  if (!dt_ok(dtype)) return refuse(PF_ERR_DTYPE, "pf_op_kv_append: dtype %d", dtype);
  if (tokens == 0 || (pages && pages->n_seqs == 0)) return PF_OK;
  if (!pages || !k || !v || !cu || !first || (rope && !pos) || (n_heads && (!q || !q_out))) return refuse(PF_ERR_NULL, "pf_op_kv_append: NULL");
  if (!n_heads && q) return refuse(PF_ERR_SHAPE, "pf_op_kv_append: q without heads");
  if (pf_status st = pages_check(dtype, pages, "pf_op_kv_append"); st != PF_OK) return st;
  const int64_t d = (int64_t)pages->kv_heads * pages->head_dim, dq = (int64_t)n_heads * pages->head_dim;
  if (!row_stride_ok(ldk, d, dtype) || !row_stride_ok(ldv, d, dtype) || !aligned(k, 16) || !aligned(v, 16) ||
      (n_heads && (!row_stride_ok(ldq, dq, dtype) || !row_stride_ok(ldqo, dq, dtype) || !aligned(q, 16) || !aligned(q_out, 16))))
    return refuse(PF_ERR_SHAPE, "pf_op_kv_append: row strides %lld, %lld for rows of %lld (q %lld, %lld for %lld), or alignment", (long long)ldk,
                  (long long)ldv, (long long)d, (long long)ldq, (long long)ldqo, (long long)dq);
  if (tokens > kMaxRows) return refuse(PF_ERR_SHAPE, "pf_op_kv_append: %d tokens are more than %d", tokens, kMaxRows);
  if (n_heads && q == q_out && ldq != ldqo) return refuse(PF_ERR_SHAPE, "pf_op_kv_append: in place with two row strides");
  if (rope)
    if (const char *w = rope_wrong(*rope, pages->head_dim)) return refuse(PF_ERR_CONFIG, "%s", w);
  RopeRows a{};
  a.dt = dtype; a.rope = rope; a.pos = pos; a.tokens = tokens; a.head_dim = pages->head_dim;
  a.q = q; a.ldq = ldq; a.q_out = q_out; a.ldqo = ldqo; a.n_heads = n_heads;
  a.k = k; a.ldk = ldk; a.v = v; a.ldv = ldv; a.kv_heads = pages->kv_heads;
  a.pages = pages_of(*pages); a.cu = cu; a.first = first; a.n_seqs = pages->n_seqs;
  return launched(launch_rope_rows(a, (hipStream_t)stream), "pf_op_kv_append");
}

// whether an attention launch of these sizes is planned at all
static bool rows_sizes_ok(int dtype, int total_q, int n_seqs, int n_heads, int kv_heads, int head_dim, int64_t max_kv) {
  return dt_ok(dtype) && total_q >= 1 && n_seqs >= 1 && head_ok(head_dim) && heads_ok(total_q, n_heads, kv_heads) && max_kv >= 1 && max_kv <= kMaxKeys;
}
static const char *rows_kernel_name(const RowsPlan &p, int dtype, int head_dim) {
  static thread_local char name[64];
  const int dim = head_dim <= 64 ? 64 : head_dim <= 96 ? 96 : 128;
  if (p.shape == ROWS_FEW) snprintf(name, sizeof(name), "attn_rows_few_kernel<%d>", dim);
  else if (p.shape == ROWS_WIDE) snprintf(name, sizeof(name), "attn_rows_wide_kernel<%d,%d>", dim, head_dim <= 80 && dim == 96 ? 5 : dim / 16);
  else snprintf(name, sizeof(name), "attn_rows_kernel<%s,%d,%s>", dtype == PF_BF16 ? "bf16" : "float", dim, p.shape == ROWS_KEYS ? "1,4" : "4,1");
  return name;
}

size_t pf_op_attention_rows_ws_bytes(int dtype, int total_q, int n_seqs, int n_heads, int kv_heads, int head_dim, int64_t max_kv) {
  if (!rows_sizes_ok(dtype, total_q, n_seqs, n_heads, kv_heads, head_dim, max_kv)) return 0;
  return rows_attention_plan(dtype, total_q, n_seqs, n_heads, kv_heads, head_dim, max_kv).ws_bytes;
}

const char *pf_attention_rows_kernel_name(int dtype, int total_q, int n_seqs, int n_heads, int kv_heads, int head_dim, int64_t max_kv,
                                          int *chunks) {
  if (!rows_sizes_ok(dtype, total_q, n_seqs, n_heads, kv_heads, head_dim, max_kv)) return "";
  const RowsPlan p = rows_attention_plan(dtype, total_q, n_seqs, n_heads, kv_heads, head_dim, max_kv);
  if (chunks) *chunks = p.splits;
  return rows_kernel_name(p, dtype, head_dim);
}

static pf_status rows_attention(RowsAttn &a, int64_t max_kv, void *ws, size_t ws_bytes, void *stream, const char *who) {
  const int64_t d = (int64_t)a.n_heads * a.head_dim;
  if (!row_stride_ok(a.ldq, d, a.dt) || !row_stride_ok(a.ldo, d, a.dt) || !aligned(a.q, 16) || !aligned(a.out, 16) || (a.lse && !aligned(a.lse, 4)))
    return refuse(PF_ERR_SHAPE, "%s: row strides %lld, %lld for rows of %lld, or alignment", who, (long long)a.ldq, (long long)a.ldo, (long long)d);
  if (a.scale <= 0.f) a.scale = 1.0f / sqrtf((float)a.head_dim);
  // the kernels take it times log2(e)
  if (!isfinite(a.scale * 1.5f)) return refuse(PF_ERR_SHAPE, "%s: scale %g", who, (double)a.scale);
  const RowsPlan p = a.mx.k_scale ? mx_attention_plan(a.dt, a.mx.format, a.total_q, a.n_seqs, a.n_heads, a.kv_heads, a.head_dim, max_kv)
                                  : rows_attention_plan(a.dt, a.total_q, a.n_seqs, a.n_heads, a.kv_heads, a.head_dim, max_kv);
  if (p.ws_bytes && (!ws || ws_bytes < p.ws_bytes || !aligned(ws, 16)))
    return refuse(PF_ERR_WORKSPACE, "%s: a 16-byte aligned workspace of %zu bytes is needed, %zu given", who, p.ws_bytes, ws ? ws_bytes : (size_t)0);
  a.ws = (float *)ws;
  // A launch has less than 2^32 threads.  The few kernel's is bounded by what is resident; it takes what pages of rows take without chunks.
  if (((int64_t)a.total_q * (a.n_heads / a.kv_heads) / 32 + a.n_seqs) * a.kv_heads * (p.shape == ROWS_FEW ? 1 : p.splits) >= (1 << 24))
    return refuse(PF_ERR_SHAPE, "%s: %d rows of %d heads in %d sequences are too many for one launch", who, a.total_q, a.n_heads, a.n_seqs);
  a.shape = p.shape;
  a.splits = p.splits;
  a.least_keys = p.least_keys;
  return launched(a.mx.k_scale ? launch_mx_attention(a, (hipStream_t)stream) : launch_rows_attention(a, (hipStream_t)stream), who);
}

pf_status pf_op_attention_packed(int dtype, const void *q, int64_t ldq, const void *k, int64_t ldk, const void *v, int64_t ldv,
                                 const int32_t *cu_q, const int32_t *cu_k, int n_seqs, int total_q, int total_k, int n_heads,
                                 int kv_heads, int head_dim, float scale, int causal, void *out, int64_t ldo, float *lse, void *ws,
                                 size_t ws_bytes, void *stream) {
  const char *who = "pf_op_attention_packed";
  if (n_seqs < 0 || total_q < 0 || total_k < 0) return refuse(PF_ERR_SHAPE, "%s: %d sequences, %d and %d rows", who, n_seqs, total_q, total_k);
  if (!dt_ok(dtype)) return refuse(PF_ERR_DTYPE, "%s: dtype %d", who, dtype);
  if (n_seqs == 0 || total_q == 0) return PF_OK;
  if (!q || !out || !cu_q || !cu_k || (total_k && (!k || !v))) return refuse(PF_ERR_NULL, "%s: NULL", who);
  if (!head_ok(head_dim) || !heads_ok(total_q, n_heads, kv_heads))
    return refuse(PF_ERR_SHAPE, "%s: %d rows, %d heads over %d of %d", who, total_q, n_heads, kv_heads, head_dim);
  if (total_k > kMaxKeys) return refuse(PF_ERR_SHAPE, "%s: %d rows of keys are more than %lld", who, total_k, (long long)kMaxKeys);
  const int64_t dk = (int64_t)kv_heads * head_dim;
  if (total_k && (!row_stride_ok(ldk, dk, dtype) || !row_stride_ok(ldv, dk, dtype) || !aligned(k, 16) || !aligned(v, 16) ||
                  ldk > (1 << 20) || ldv > (1 << 20)))   // a tile's rows are addressed by 32-bit offsets
    return refuse(PF_ERR_SHAPE, "%s: row strides %lld, %lld for rows of %lld (at most 2^20), or alignment", who, (long long)ldk, (long long)ldv, (long long)dk);
  RowsAttn a{};
  a.dt = dtype; a.q = q; a.ldq = ldq; a.k = k; a.ldk = ldk; a.v = v; a.ldv = ldv; a.cu_q = cu_q; a.cu_k = cu_k;
  a.n_seqs = n_seqs; a.total_q = total_q; a.total_k = total_k; a.n_heads = n_heads; a.kv_heads = kv_heads; a.head_dim = head_dim;
  a.scale = scale; a.causal = causal != 0; a.out = out; a.ldo = ldo; a.lse = lse;
  return rows_attention(a, total_k > 0 ? total_k : 1, ws, ws_bytes, stream, who);
}

pf_status pf_op_attention_paged(int dtype, const void *q, int64_t ldq, const pf_kv_pages *pages, const int32_t *cu_q,
                                const int32_t *first, const int32_t *kv_len, int total_q, int n_heads, float scale, int causal,
                                void *out, int64_t ldo, float *lse, void *ws, size_t ws_bytes, void *stream) {
  const char *who = "pf_op_attention_paged";
  if (total_q < 0) return refuse(PF_ERR_SHAPE, "%s: %d rows", who, total_q);
  if (!dt_ok(dtype)) return refuse(PF_ERR_DTYPE, "%s: dtype %d", who, dtype);
  if (total_q == 0 || (pages && pages->n_seqs == 0)) return PF_OK;
  if (!pages || !q || !out || !cu_q || !kv_len || (causal && !first)) return refuse(PF_ERR_NULL, "%s: NULL", who);
  if (pf_status st = pages_check(dtype, pages, who); st != PF_OK) return st;
  if (!heads_ok(total_q, n_heads, pages->kv_heads))
    return refuse(PF_ERR_SHAPE, "%s: %d rows, %d heads over %d", who, total_q, n_heads, pages->kv_heads);
  const int64_t max_kv = (int64_t)pages->max_pages * pages->page_size;
  if (max_kv > kMaxKeys) return refuse(PF_ERR_SHAPE, "%s: max_pages * page_size = %lld", who, (long long)max_kv);
  RowsAttn a{};
  a.dt = dtype; a.q = q; a.ldq = ldq; a.pages = pages_of(*pages); a.cu_q = cu_q; a.first = causal ? first : nullptr; a.kv_len = kv_len;
  a.n_seqs = pages->n_seqs; a.total_q = total_q; a.n_heads = n_heads; a.kv_heads = pages->kv_heads; a.head_dim = pages->head_dim;
  a.scale = scale; a.causal = causal != 0; a.out = out; a.ldo = ldo; a.lse = lse;
  return rows_attention(a, max_kv, ws, ws_bytes, stream, who);
}

pf_status pf_op_norm_residual(int dtype, const void *y, int64_t ldy, const pf_norm *post, const float *gate, int64_t gate_stride,
                              int gate_tanh, float x_scale, const float *x, int64_t ldx, float *x_out, int64_t ldxo,
                              const pf_norm *pre, const float *shift, const float *scale, int64_t mod_stride, void *h,
                              int64_t ldh, const int32_t *cu, int n_seqs, int rows, int d, void *stream) {
  const char *who = "pf_op_norm_residual";
  if (rows < 0 || n_seqs < 0) return refuse(PF_ERR_SHAPE, "%s: %d rows, %d sequences", who, rows, n_seqs);
  if (!dt_ok(dtype)) return refuse(PF_ERR_DTYPE, "%s: dtype %d", who, dtype);
  if (rows == 0 || (cu && n_seqs == 0)) return PF_OK;
  if (!x || (!x_out && !h)) return refuse(PF_ERR_NULL, "%s: x, or both outputs", who);
  const size_t al = dtype == PF_BF16 ? 8 : 16;
  if (cu && n_seqs > kMaxSeqs) return refuse(PF_ERR_SHAPE, "%s: %d sequences are more than %d", who, n_seqs, kMaxSeqs);
  if (rows > kMaxRows) return refuse(PF_ERR_SHAPE, "%s: %d rows are more than %d", who, rows, kMaxRows);
  if (d < 8 || d % 8 || d > 8192) return refuse(PF_ERR_SHAPE, "%s: d = %d", who, d);
  if (ldx < d || ldx % 4 || !aligned(x, 16) || (y && (ldy < d || ldy % 4 || !aligned(y, al))) ||
      (x_out && (ldxo < d || ldxo % 4 || !aligned(x_out, 16))) || (h && (ldh < d || ldh % 4 || !aligned(h, al))) ||
      (gate && !aligned(gate, 16)) || (scale && !aligned(scale, 16)) || (shift && !aligned(shift, 16)))
    return refuse(PF_ERR_SHAPE, "%s: row strides or alignment (d = %d)", who, d);
  if (cu && ((gate && gate_stride % 4) || ((scale || shift) && mod_stride % 4)))
    return refuse(PF_ERR_SHAPE, "%s: strides of the vectors per sequence must be multiples of 4", who);
  if ((x_out == x && ldxo != ldx) || (h && h == y && ldh != ldy)) return refuse(PF_ERR_SHAPE, "%s: in place with two row strides", who);
  NormResidual a{};
  const pf_norm *sides[2] = {post, pre};
  for (int i = 0; i < 2; ++i) {
    if (!sides[i]) continue;
    const pf_norm &n = *sides[i];
    if (n.kind < PF_NORM_NONE || n.kind > PF_NORM_LAYER) return refuse(PF_ERR_CONFIG, "%s: norm kind %d", who, n.kind);
    if (n.kind != PF_NORM_NONE && !(n.eps >= 0.f)) return refuse(PF_ERR_CONFIG, "%s: norm eps", who);
    if (!aligned(n.weight, al) || !aligned(n.bias, al)) return refuse(PF_ERR_SHAPE, "%s: alignment of norm weights", who);
    if (n.kind == PF_NORM_NONE && (n.weight || n.bias)) return refuse(PF_ERR_CONFIG, "%s: weights of a norm of kind NONE", who);
    (i ? a.pre : a.post) = NormSide{n.kind, n.eps, n.weight, n.bias};
  }
  a.dt = dtype; a.y = y; a.ldy = ldy; a.gate = gate; a.gate_stride = gate_stride; a.gate_tanh = gate_tanh != 0; a.x_scale = x_scale;
  a.x = x; a.ldx = ldx; a.x_out = x_out; a.ldxo = ldxo; a.shift = shift; a.scale = scale; a.mod_stride = mod_stride; a.h = h; a.ldh = ldh;
  a.cu = cu; a.n_seqs = n_seqs; a.rows = rows; a.d = d;
  return launched(launch_norm_residual(a, (hipStream_t)stream), who);
}

int pf_kv_mx_row_bytes(int format, int head_dim) {
  return (format == PF_MX_E4M3 || format == PF_MX_E2M1) && head_ok(head_dim) ? mx_row_bytes(format, head_dim) : 0;
}

pf_status pf_op_qk_norm_rope(int dtype, const void *q, int64_t ldq, const pf_norm *q_norm, void *q_out, int64_t ldqo, int n_heads,
                             const void *k, int64_t ldk, const pf_norm *k_norm, void *k_out, int64_t ldko, int kv_heads,
                             const pf_rope *rope, const int32_t *pos, int tokens, int head_dim, void *stream) {
  const char *who = "pf_op_qk_norm_rope";
  if (tokens < 0 || n_heads < 0 || n_heads > 65536 || kv_heads < 0 || kv_heads > 65536)
    return refuse(PF_ERR_SHAPE, "%s: %d tokens, %d and %d heads", who, tokens, n_heads, kv_heads);
  if (!dt_ok(dtype)) return refuse(PF_ERR_DTYPE, "%s: dtype %d", who, dtype);
  if (tokens == 0 || n_heads + kv_heads == 0) return PF_OK;
  if ((n_heads && (!q || !q_out)) || (kv_heads && (!k || !k_out)) || (rope && !pos)) return refuse(PF_ERR_NULL, "%s: NULL", who);
  if (!head_ok(head_dim)) return refuse(PF_ERR_SHAPE, "%s: heads of %d", who, head_dim);
  const int64_t dq = (int64_t)n_heads * head_dim, dk = (int64_t)kv_heads * head_dim;
  if ((n_heads && (!row_stride_ok(ldq, dq, dtype) || !row_stride_ok(ldqo, dq, dtype) || !aligned(q, 16) || !aligned(q_out, 16))) ||
      (kv_heads && (!row_stride_ok(ldk, dk, dtype) || !row_stride_ok(ldko, dk, dtype) || !aligned(k, 16) || !aligned(k_out, 16))) ||
      (rope && !aligned(pos, 4)))
    return refuse(PF_ERR_SHAPE, "%s: row strides %lld, %lld for rows of %lld (k %lld, %lld for %lld), or alignment", who, (long long)ldq, (long long)ldqo,
                  (long long)dq, (long long)ldk, (long long)ldko, (long long)dk);
  if (tokens > kMaxRows) return refuse(PF_ERR_SHAPE, "%s: %d tokens are more than %d", who, tokens, kMaxRows);
  if ((n_heads && q == q_out && ldq != ldqo) || (kv_heads && k == k_out && ldk != ldko)) return refuse(PF_ERR_SHAPE, "%s: in place with two row strides", who);
  if (rope)
    if (const char *w = rope_wrong(*rope, head_dim)) return refuse(PF_ERR_CONFIG, "%s", w);
  HeadRows a{};
  if (pf_status st = head_norm(n_heads ? q_norm : nullptr, a.norm[0], who); st != PF_OK) return st;
  if (pf_status st = head_norm(kv_heads ? k_norm : nullptr, a.norm[1], who); st != PF_OK) return st;
  a.dt = dtype; a.q = q; a.ldq = ldq; a.q_out = q_out; a.ldqo = ldqo; a.n_heads = n_heads;
  a.k = k; a.ldk = ldk; a.k_out = k_out; a.ldko = ldko; a.kv_heads = kv_heads;
  a.pos = pos; a.tokens = tokens; a.head_dim = head_dim;
  return launched(launch_head_rows(a, rope, (hipStream_t)stream), who);
}

pf_status pf_op_kv_append_mx(int dtype, const pf_kv_mx_pages *pages, const void *k, int64_t ldk, const pf_norm *k_norm, const void *v,
                             int64_t ldv, const int32_t *cu, const int32_t *first, int tokens, const pf_rope *rope, const int32_t *pos,
                             const void *q, int64_t ldq, const pf_norm *q_norm, void *q_out, int64_t ldqo, int n_heads, void *stream) {
  const char *who = "pf_op_kv_append_mx";
  if (tokens < 0 || n_heads < 0 || n_heads > 65536) return refuse(PF_ERR_SHAPE, "%s: %d tokens, %d heads", who, tokens, n_heads);
  if (!dt_ok(dtype)) return refuse(PF_ERR_DTYPE, "%s: dtype %d", who, dtype);
  if (tokens == 0 || (pages && pages->n_seqs == 0)) return PF_OK;
  if (!pages || !k || !v || !cu || !first || (rope && !pos) || (n_heads && (!q || !q_out))) return refuse(PF_ERR_NULL, "%s: NULL", who);
  if (!n_heads && q) return refuse(PF_ERR_SHAPE, "%s: q without heads", who);
  if (pf_status st = mx_pages_check(pages, who); st != PF_OK) return st;
  const int64_t d = (int64_t)pages->kv_heads * pages->head_dim, dq = (int64_t)n_heads * pages->head_dim;
  if (!row_stride_ok(ldk, d, dtype) || !row_stride_ok(ldv, d, dtype) || !aligned(k, 16) || !aligned(v, 16) || (rope && !aligned(pos, 4)) ||
      (n_heads && (!row_stride_ok(ldq, dq, dtype) || !row_stride_ok(ldqo, dq, dtype) || !aligned(q, 16) || !aligned(q_out, 16))))
    return refuse(PF_ERR_SHAPE, "%s: row strides %lld, %lld for rows of %lld (q %lld, %lld for %lld), or alignment", who, (long long)ldk, (long long)ldv,
                  (long long)d, (long long)ldq, (long long)ldqo, (long long)dq);
  if (tokens > kMaxRows) return refuse(PF_ERR_SHAPE, "%s: %d tokens are more than %d", who, tokens, kMaxRows);
  if (n_heads && q == q_out && ldq != ldqo) return refuse(PF_ERR_SHAPE, "%s: in place with two row strides", who);
  if (rope)
    if (const char *w = rope_wrong(*rope, pages->head_dim)) return refuse(PF_ERR_CONFIG, "%s", w);
  HeadRows a{};
  if (pf_status st = head_norm(n_heads ? q_norm : nullptr, a.norm[0], who); st != PF_OK) return st;
  if (pf_status st = head_norm(k_norm, a.norm[1], who); st != PF_OK) return st;
  a.dt = dtype; a.q = q; a.ldq = ldq; a.q_out = q_out; a.ldqo = ldqo; a.n_heads = n_heads;
  a.k = k; a.ldk = ldk; a.v = v; a.ldv = ldv; a.kv_heads = pages->kv_heads;
  a.pos = pos; a.tokens = tokens; a.head_dim = pages->head_dim;
  a.pages = mx_places(*pages); a.mx = mx_numbers(*pages); a.cu = cu; a.first = first; a.n_seqs = pages->n_seqs;
  return launched(launch_head_rows(a, rope, (hipStream_t)stream), who);
}

pf_status pf_op_kv_read_mx(int dtype, const pf_kv_mx_pages *pages, const int32_t *cu, const int32_t *first, int tokens, void *k_out,
                           int64_t ldk, void *v_out, int64_t ldv, void *stream) {
  const char *who = "pf_op_kv_read_mx";
  if (tokens < 0) return refuse(PF_ERR_SHAPE, "%s: %d tokens", who, tokens);
  if (!dt_ok(dtype)) return refuse(PF_ERR_DTYPE, "%s: dtype %d", who, dtype);
  if (tokens == 0 || (pages && pages->n_seqs == 0)) return PF_OK;
  if (!pages || !cu || !first || (!k_out && !v_out)) return refuse(PF_ERR_NULL, "%s: NULL", who);
  if (pf_status st = mx_pages_check(pages, who); st != PF_OK) return st;
  const int64_t d = (int64_t)pages->kv_heads * pages->head_dim;
  if ((k_out && (!row_stride_ok(ldk, d, dtype) || !aligned(k_out, 16))) || (v_out && (!row_stride_ok(ldv, d, dtype) || !aligned(v_out, 16))))
    return refuse(PF_ERR_SHAPE, "%s: row strides %lld, %lld for rows of %lld, or alignment", who, (long long)ldk, (long long)ldv, (long long)d);
  if (tokens > kMaxRows) return refuse(PF_ERR_SHAPE, "%s: %d tokens are more than %d", who, tokens, kMaxRows);
  MxRead a{};
  a.dt = dtype; a.pages = mx_places(*pages); a.mx = mx_numbers(*pages); a.cu = cu; a.first = first; a.n_seqs = pages->n_seqs;
  a.tokens = tokens; a.kv_heads = pages->kv_heads; a.head_dim = pages->head_dim; a.k_out = k_out; a.ldk = ldk; a.v_out = v_out; a.ldv = ldv;
  return launched(launch_mx_read(a, (hipStream_t)stream), who);
}

size_t pf_op_attention_mx_ws_bytes(int dtype, int format, int total_q, int n_seqs, int n_heads, int kv_heads, int head_dim, int64_t max_kv) {
  if ((format != PF_MX_E4M3 && format != PF_MX_E2M1) || !rows_sizes_ok(dtype, total_q, n_seqs, n_heads, kv_heads, head_dim, max_kv)) return 0;
  return mx_attention_plan(dtype, format, total_q, n_seqs, n_heads, kv_heads, head_dim, max_kv).ws_bytes;
}

const char *pf_attention_mx_kernel_name(int dtype, int format, int total_q, int n_seqs, int n_heads, int kv_heads, int head_dim,
                                        int64_t max_kv, int *chunks) {
  if ((format != PF_MX_E4M3 && format != PF_MX_E2M1) || !rows_sizes_ok(dtype, total_q, n_seqs, n_heads, kv_heads, head_dim, max_kv)) return "";
  const RowsPlan p = mx_attention_plan(dtype, format, total_q, n_seqs, n_heads, kv_heads, head_dim, max_kv);
  if (chunks) *chunks = p.splits;
  return rows_kernel_name(p, dtype, head_dim);
}

pf_status pf_op_attention_mx(int dtype, const void *q, int64_t ldq, const pf_kv_mx_pages *pages, const int32_t *cu_q,
                             const int32_t *first, const int32_t *kv_len, int total_q, int n_heads, float scale, int causal, void *out,
                             int64_t ldo, float *lse, void *ws, size_t ws_bytes, void *stream) {
  const char *who = "pf_op_attention_mx";
  if (total_q < 0) return refuse(PF_ERR_SHAPE, "%s: %d rows", who, total_q);
  if (!dt_ok(dtype)) return refuse(PF_ERR_DTYPE, "%s: dtype %d", who, dtype);
  if (total_q == 0 || (pages && pages->n_seqs == 0)) return PF_OK;
  if (!pages || !q || !out || !cu_q || !kv_len || (causal && !first)) return refuse(PF_ERR_NULL, "%s: NULL", who);
  if (pf_status st = mx_pages_check(pages, who); st != PF_OK) return st;
  if (!heads_ok(total_q, n_heads, pages->kv_heads))
    return refuse(PF_ERR_SHAPE, "%s: %d rows, %d heads over %d", who, total_q, n_heads, pages->kv_heads);
  const int64_t max_kv = (int64_t)pages->max_pages * pages->page_size;
  if (max_kv > kMaxKeys) return refuse(PF_ERR_SHAPE, "%s: max_pages * page_size = %lld", who, (long long)max_kv);
  RowsAttn a{};
  a.dt = dtype; a.q = q; a.ldq = ldq; a.pages = mx_places(*pages); a.mx = mx_numbers(*pages); a.cu_q = cu_q; a.first = causal ? first : nullptr;
  a.kv_len = kv_len; a.n_seqs = pages->n_seqs; a.total_q = total_q; a.n_heads = n_heads; a.kv_heads = pages->kv_heads; a.head_dim = pages->head_dim;
  a.scale = scale; a.causal = causal != 0; a.out = out; a.ldo = ldo; a.lse = lse;
  return rows_attention(a, max_kv, ws, ws_bytes, stream, who);
}

}  // extern "C"
