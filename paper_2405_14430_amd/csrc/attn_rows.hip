// Attention of packed query rows over packed keys or over pages: plain kernel, one wave per query row and head.
// A lane scores one key of a block of 64, the running maximum and sum are kept in 32 bits, and the weighted sum of the values
// goes key by key with the lanes along the channels.
#include "requests.h"

namespace pf {
namespace {

template <typename T, bool PAGED>
__global__ __launch_bounds__(256) void attn_rows_plain_kernel(RowsAttn a) {
  __shared__ float qs[4][128];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t id = (int64_t)blockIdx.x * 4 + wave;
  if (id >= (int64_t)a.total_q * a.n_heads) return;
  const int row = (int)(id / a.n_heads), h = (int)(id % a.n_heads), hk = h / (a.n_heads / a.kv_heads), dh = a.head_dim;
  const int s = wave_search(a.n_seqs, lane, row, [&](int i) { return a.cu_q[i]; });
  if (s < 0 || s >= a.n_seqs) return;
  int q0, q1, k0 = 0, kn;
  sequence_rows(a.cu_q, s, a.total_q, q0, q1);
  const int i = row - q0;
  int64_t last;   // one past the last key the row sees
  if (PAGED) {
    kn = clampi(a.kv_len[s], 0, a.pages.max_pages << a.pages.page_shift);
    last = a.causal ? (int64_t)a.first[s] + i + 1 : kn;
  } else {
    int k1;
    sequence_rows(a.cu_k, s, a.total_k, k0, k1);
    kn = k1 - k0;
    last = a.causal ? (int64_t)i + kn - (q1 - q0) + 1 : kn;
  }
  if (last > kn) last = kn;
  const T *q = (const T *)a.q + row * a.ldq + h * dh;
  for (int c = lane; c < dh; c += 64) qs[wave][c] = to_f32(q[c]) * a.scale;
  __builtin_amdgcn_wave_barrier();
  // start of key j's row of this head, nullptr where its page is none
  auto key_row = [&](int j, bool value) -> const T * {
    if (!PAGED) return value ? (const T *)a.v + (int64_t)(k0 + j) * a.ldv + hk * dh : (const T *)a.k + (int64_t)(k0 + j) * a.ldk + hk * dh;
    const int page = a.pages.table[(int64_t)s * a.pages.max_pages + (j >> a.pages.page_shift)];
    if (page < 0 || page >= a.pages.n_pages) return nullptr;
    const int64_t at = (((int64_t)hk << a.pages.page_shift) + (j & ((1 << a.pages.page_shift) - 1))) * dh;
    return value ? (const T *)a.pages.v + page * a.pages.v_stride + at : (const T *)a.pages.k + page * a.pages.k_stride + at;
  };
  float m = -INFINITY, l = 0.f, o[2] = {0.f, 0.f};
  for (int j0 = 0; j0 < last; j0 += 64) {
    const int j = j0 + lane;
    float sc = -INFINITY;
    if (j < last) {
      if (const T *kr = key_row(j, false)) {
        sc = 0.f;
        for (int c = 0; c < dh; ++c) sc = fmaf(qs[wave][c], to_f32(kr[c]), sc);
      }
    }
    const float mn = fmaxf(m, wave_max(sc));
    if (mn == -INFINITY) continue;
    const float keep = expf(m - mn), p = expf(sc - mn);
    l = l * keep + wave_sum(p);
    o[0] *= keep;
    o[1] *= keep;
    m = mn;
    const int n = (int)(last - j0 < 64 ? last - j0 : 64);
    for (int e = 0; e < n; ++e) {
      const T *vr = key_row(j0 + e, true);
      if (!vr) continue;
      const float w = __shfl(p, e, kWave);
      if (lane < dh) o[0] = fmaf(w, to_f32(vr[lane]), o[0]);
      if (lane + 64 < dh) o[1] = fmaf(w, to_f32(vr[lane + 64]), o[1]);
    }
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  T *op = (T *)a.out + row * a.ldo + h * dh;
  if (lane < dh) op[lane] = from_f32<T>(o[0] * inv);
  if (lane + 64 < dh) op[lane + 64] = from_f32<T>(o[1] * inv);
  if (a.lse && lane == 0) a.lse[(int64_t)row * a.n_heads + h] = l > 0.f ? m + logf(l) : -INFINITY;
}

}  // namespace

RowsPlan rows_attention_plan(int, int, int, int, int, int, int64_t) { return RowsPlan{4, 1, 0}; }

hipError_t launch_rows_attention(const RowsAttn &a, hipStream_t s) {
  const int64_t n = (int64_t)a.total_q * a.n_heads;
  const dim3 g((unsigned)((n + 3) / 4));
  const bool paged = a.pages.table != nullptr;
  if (a.dt == DT_BF16 && paged) attn_rows_plain_kernel<bf16_t, true><<<g, 256, 0, s>>>(a);
  else if (a.dt == DT_BF16) attn_rows_plain_kernel<bf16_t, false><<<g, 256, 0, s>>>(a);
  else if (paged) attn_rows_plain_kernel<float, true><<<g, 256, 0, s>>>(a);
  else attn_rows_plain_kernel<float, false><<<g, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace pf
