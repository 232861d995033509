// Shared pieces of the operators on packed rows: rows of several sequences behind each other, cu[s] .. cu[s + 1] those of
// sequence s, and keys / values in pages that a table assigns to sequences.  Lengths, positions and tables are device
// memory that the host never sees, so every kernel bounds what it reads from them before it uses it as an address.
#pragma once
#include "../../include/pfstage.h"
#include "common.h"
#include "ops.h"

namespace pf {

pf_status note_error(pf_status st, const char *text);   // what pf_last_error(NULL) returns next on this thread (stage.hip)

// The largest s in [0, n] with key(s) <= x for a non-decreasing key, found by the 64 lanes of a wave together: each round
// probes 64 evenly spaced places at once, so 64 entries take one memory latency and 4096 two.  Returns -1 if key(0) > x.
// Keys that decrease somewhere give some s in [-1, n] all the same.  n is at most 2^30: places behind it are counted in 32 bits.
template <typename F>
__device__ __forceinline__ int wave_search(int n, int lane, int64_t x, F &&key) {
  int lo = -1, hi = n + 1;                  // key(lo) <= x < key(hi)
  while (hi - lo > 1) {
    const int step = (hi - lo - 1 + 63) >> 6;
    const int at = lo + 1 + lane * step;
    const bool le = at < hi && (int64_t)key(at) <= x;
    const int cnt = __builtin_popcountll(__builtin_amdgcn_ballot_w64(le));
    if (cnt == 0) { hi = lo + 1; break; }
    lo += 1 + (cnt - 1) * step;
    hi = lo + step < hi ? lo + step : hi;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }

// Rows [begin, end) of sequence s, inside [0, total] whatever cu holds.
__device__ __forceinline__ void sequence_rows(const int32_t *cu, int s, int total, int &begin, int &end) {
  begin = clampi(cu[s], 0, total);
  end = clampi(cu[s + 1], begin, total);
}

// What a kernel needs of pf_kv_pages: page p of K starts p * k_stride elements in and holds [kv_heads][1 << page_shift][head_dim].
struct Pages {
  void *k, *v;
  int64_t k_stride, v_stride;
  const int32_t *table;
  int n_pages, page_shift, max_pages;
};
inline Pages pages_of(const pf_kv_pages &p) {
  return Pages{p.k, p.v, p.k_page_stride, p.v_page_stride, p.table, p.n_pages, __builtin_ctz((unsigned)p.page_size), p.max_pages};
}

// Pages of 8- or 4-bit numbers: `pages` has bytes and strides in bytes; a row of a head is row_bytes of codes and, in arrays of their own,
// `blocks` exponents.  No scales: pages of rows.
struct MxPages {
  int format, row_bytes, blocks;
  uint8_t *k_scale, *v_scale;
  int64_t k_scale_stride, v_scale_stride;
};

// Calls that move more bytes than the 256 MiB cache in front of the memory holds read their rows with non-temporal loads, which do not
// push out what is being written; smaller ones find rows there that the kernel before has left, and lose by it (append of 16384 rows
// of 32 + 2 x 8 heads of 128, bf16, 400 MB: 81 -> 66 us, 8192 rows 34 -> 37; norm of 8192 rows of 4096, bf16, 403 MB:
// 120 -> 109, 16384 rows of 1152, 226 MB: 48 -> 55; the same rows again and again).
constexpr int64_t kReadOnceBytes = 256ll << 20;

// Rows of one launch of the row kernels, whose workgroups of up to 512 threads take a row each: a launch has less than 2^32 threads.
constexpr int kLaunchRows = 1 << 22;

struct RopeRows {
  int dt;
  const pf_rope *rope;   // nullptr: rows are copied (append only)
  const int32_t *pos;
  int tokens, head_dim;
  const void *q; int64_t ldq; void *q_out; int64_t ldqo; int n_heads;     // rotated rows (q of an append; may have no heads)
  const void *k; int64_t ldk; const void *v; int64_t ldv; int kv_heads;   // append only
  Pages pages;
  const int32_t *cu, *first;
  int n_seqs;            // 0: no append
};
hipError_t launch_rope_rows(const RopeRows &a, hipStream_t s);

struct NormSide { int kind; float eps; const void *weight, *bias; };
struct NormResidual {
  int dt;
  const void *y; int64_t ldy;
  NormSide post, pre;
  const float *gate; int64_t gate_stride; int gate_tanh;
  float x_scale;
  const float *x; int64_t ldx;
  float *x_out; int64_t ldxo;
  const float *shift, *scale; int64_t mod_stride;
  void *h; int64_t ldh;
  const int32_t *cu; int n_seqs;
  int rows, d;
  int row0;                // first row of the launch (set there)
  bool once;               // x and y are read with non-temporal loads (set at the launch)
};
hipError_t launch_norm_residual(const NormResidual &a, hipStream_t s);

// Heads of q and k normed and turned; with n_seqs, k and v go into pages of few bits (k_out, ldko are not used then).
struct HeadRows {
  int dt;
  const void *q; int64_t ldq; void *q_out; int64_t ldqo; int n_heads;
  const void *k; int64_t ldk; void *k_out; int64_t ldko; int kv_heads;
  const void *v; int64_t ldv;
  NormSide norm[2];        // of q and of k
  const int32_t *pos;
  int tokens, head_dim;
  Pages pages;             // strides in bytes
  MxPages mx;
  const int32_t *cu, *first;
  int n_seqs;              // 0: no pages
};
hipError_t launch_head_rows(const HeadRows &a, const pf_rope *rope, hipStream_t s);

// Slots of pages of few bits to rows; k_out or v_out may be nullptr.
struct MxRead {
  int dt;
  Pages pages;             // strides in bytes
  MxPages mx;
  const int32_t *cu, *first;
  int n_seqs, tokens, kv_heads, head_dim;
  void *k_out; int64_t ldk; void *v_out; int64_t ldv;
};
hipError_t launch_mx_read(const MxRead &a, hipStream_t s);

// Attention of packed query rows over packed keys (pages.k == nullptr) or over pages.
struct RowsAttn {
  int dt;
  const void *q; int64_t ldq;
  const void *k; int64_t ldk; const void *v; int64_t ldv;   // packed keys: rows cu_k[s] .. cu_k[s + 1]
  Pages pages;                                              // paged keys: slots [0, kv_len[s])
  MxPages mx;                                               // pages.k and pages.v hold its numbers (launch_mx_attention)
  const int32_t *cu_q, *cu_k, *first, *kv_len;
  int n_seqs, total_q, total_k;
  int n_heads, kv_heads, head_dim;
  float scale;
  int causal;
  void *out; int64_t ldo;
  float *lse;
  float *ws;
  int shape, splits, least_keys;       // of the plan
};
enum { ROWS_TILES, ROWS_WIDE, ROWS_KEYS, ROWS_FEW };   // kernels of attn_rows.h; the last one of attn_rows_mx.hip
struct RowsPlan { int shape, splits, least_keys; size_t ws_bytes; };   // splits: chunks of the keys, none smaller than least_keys
RowsPlan rows_attention_plan(int dt, int total_q, int n_seqs, int n_heads, int kv_heads, int head_dim, int64_t max_kv);
RowsPlan mx_attention_plan(int dt, int format, int total_q, int n_seqs, int n_heads, int kv_heads, int head_dim, int64_t max_kv);
hipError_t launch_rows_attention(const RowsAttn &a, hipStream_t s);
hipError_t launch_mx_attention(const RowsAttn &a, hipStream_t s);
hipError_t launch_rows_join(const RowsAttn &a, hipStream_t s);   // of the partial results in a.ws

}  // namespace pf
