// Attention of packed rows over rows and over pages of rows (kernels: attn_rows.h), the join of their chunks, and the plan of a launch.
#include "attn_rows.h"

namespace pf {
namespace {

// Joins the chunks of a row: out = sum 2^(m_c - m) O_c / sum 2^(m_c - m) l_c, W waves per (token, head).  A thread sums four channels of
// every GROUPS-th chunk, the groups are added up through LDS in their order.  Chunks that saw no key of the row left l = 0; their O is
// not used.  One whose weight is 0 only in 32 bits is: its infinities and NaN reach the row, as they do where the keys are one chunk.  Four to five microseconds, launch included, of three memory latencies behind each other, for a token of 16 heads in 128
// chunks as for 64 of 32 heads in 8.
template <typename T, int W>
__global__ __launch_bounds__(256) void attn_rows_join_kernel(RowsAttn a) {
  constexpr int R = 4 / W, NT = 64 * W;                       // rows per workgroup, threads per row
  __shared__ float weight[R][kMaxChunks], part[R][NT * 4], stat[R][2 * W];
  const int slot = threadIdx.x / NT, tid = threadIdx.x % NT, lane = threadIdx.x & 63, wave = tid >> 6;
  const int dh = a.head_dim;
  const int64_t all = (int64_t)a.total_q * a.n_heads;
  const int64_t id = (int64_t)blockIdx.x * R + slot;
  const int row = (int)(min(id, all - 1) / a.n_heads), head = (int)(min(id, all - 1) - (int64_t)row * a.n_heads);
  const bool live = id < all && row >= a.cu_q[0] && row < a.cu_q[a.n_seqs];
  const float2 *ml = reinterpret_cast<const float2 *>(a.ws + (int64_t)a.splits * all * dh) + id;
  constexpr int PER = (kMaxChunks + NT - 1) / NT;
  constexpr float kNone = -1.f;                               // in place of a weight: no key
  float2 v[PER];
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    v[i] = make_float2(-INFINITY, 0.f);
    if (live && i * NT + tid < a.splits) v[i] = ml[(i * NT + tid) * all];
    m = fmaxf(m, v[i].x);
  }
  m = wave_max(m);
  if (lane == 0) stat[slot][wave] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < W; ++i) m = fmaxf(m, stat[slot][i]);
  float l = 0.f;
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (i * NT + tid < a.splits) {
      const float w = v[i].y != 0.f ? __builtin_amdgcn_exp2f(v[i].x - m) : kNone;
      weight[slot][i * NT + tid] = w;
      if (w != kNone) l = fmaf(w, v[i].y, l);
    }
  l = wave_sum(l);
  if (lane == 0) stat[slot][W + wave] = l;
  __syncthreads();
  l = 0.f;
#pragma unroll
  for (int i = 0; i < W; ++i) l += stat[slot][W + i];
  const int cl = dh <= 64 ? 16 : 32, groups = NT / cl;        // threads across a row's channels
  const int c = tid % cl * 4, g = tid / cl;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  if (live && c < dh) {
    // eight chunks' loads at a time, whether they count or not (a chunk that does not may hold anything)
    for (int i0 = g; i0 < a.splits; i0 += 8 * groups) {
      float4 x[8];
      float w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int i = min(i0 + j * groups, a.splits - 1);
        x[j] = *reinterpret_cast<const float4 *>(a.ws + ((int64_t)i * all + id) * dh + c);
        w[j] = i0 + j * groups < a.splits ? weight[slot][i] : kNone;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (w[j] != kNone) acc = make_float4(fmaf(w[j], x[j].x, acc.x), fmaf(w[j], x[j].y, acc.y), fmaf(w[j], x[j].z, acc.z), fmaf(w[j], x[j].w, acc.w));
    }
  }
  *reinterpret_cast<float4 *>(&part[slot][tid * 4]) = acc;
  __syncthreads();
  if (!live) return;
  const float inv = l != 0.f ? 1.f / l : 0.f;
  if (g == 0 && c < dh) {
    for (int i = 1; i < groups; ++i) {
      const float4 x = *reinterpret_cast<const float4 *>(&part[slot][(i * cl + tid) * 4]);
      acc = make_float4(acc.x + x.x, acc.y + x.y, acc.z + x.z, acc.w + x.w);
    }
    T *dst = (T *)a.out + (int64_t)row * a.ldo + (int64_t)head * dh + c;
    if constexpr (sizeof(T) == 4) *reinterpret_cast<float4 *>(dst) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
    else *reinterpret_cast<bf16x4 *>(dst) = bf16x4{(bf16_t)(acc.x * inv), (bf16_t)(acc.y * inv), (bf16_t)(acc.z * inv), (bf16_t)(acc.w * inv)};
  }
  if (a.lse && tid == 0) a.lse[id] = l != 0.f ? m * kLn2 + logf(l) : -INFINITY;
}

template <typename T>
hipError_t launch_join(const RowsAttn &a, hipStream_t s) {
  const int64_t all = (int64_t)a.total_q * a.n_heads;
  // four waves per row where a wave would have more than eight chunks to add up per thread (128 chunks of a token of 16 heads: the call
  // takes 30.9 us, with one wave 34.4; 16 chunks of 64 tokens of 32 heads: 176, with four waves 180)
  if (a.splits > 16) attn_rows_join_kernel<T, 4><<<dim3((unsigned)all), 256, 0, s>>>(a);
  else attn_rows_join_kernel<T, 1><<<dim3((unsigned)((all + 3) / 4)), 256, 0, s>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_type(const RowsAttn &a, hipStream_t s) {
  if (a.pages.table) return a.causal ? launch_dim<T, KEYS_PAGES, true>(a, s) : launch_dim<T, KEYS_PAGES, false>(a, s);
  return a.causal ? launch_dim<T, KEYS_PACKED, true>(a, s) : launch_dim<T, KEYS_PACKED, false>(a, s);
}

}  // namespace

// Which kernel, and how many chunks of the key range, by the estimated time in microseconds.  The lengths are on the device: the host
// knows the rows of all sequences, their number, and that none has more than max_kv keys; a causal mask and shorter
// sequences make all the estimates too long alike.
RowsPlan rows_attention_plan(int dt, int total_q, int n_seqs, int n_heads, int kv_heads, int head_dim, int64_t max_kv) {
  const int64_t rows = (int64_t)total_q * (n_heads / kv_heads), tiles = (max_kv + 63) / 64;
  const auto wgs = [&](int per) { return workgroups(total_q, n_heads / kv_heads, n_seqs, kv_heads, per); };
  const auto rounds = [](int64_t n, int fit) { return n <= 2 * fit ? (double)((n + fit - 1) / fit) : (double)n / fit + 0.5; };
  // the second launch, and the partial results on their way through memory (4 TB/s)
  const double row_us = (double)total_q * n_heads * head_dim * 4.9e-7;
  const auto join_us = [&](int64_t n) { return n > 1 ? 4.0 + (4 * n + 2) * row_us : 0.0; };
  const int dim = head_dim <= 64 ? 0 : head_dim <= 96 ? 1 : 2;

  RowsPlan p{ROWS_TILES, 1, 0, 0};
  double best = 1e300;
  const auto offer = [&](int shape, int64_t n, double us) {
    if (us < best - 1e-9) {
      best = us;
      p = RowsPlan{shape, (int)n, 256, 0};
    }
  };
  // chunks of four tiles or more, and none for launches that fill the chip twice without
  const int64_t most = tiles < 8 ? 1 : tiles / 4 < 16 ? tiles / 4 : 16;
  for (int64_t n = 1; n <= most; ++n) {
    const double steps = (double)((tiles + n - 1) / n);
    // 128 rows: two workgroups fit a CU; a tile of 64 keys takes this long where a CU has one, and where it has two (head sizes 64, 96, 128)
    constexpr double kOne[] = {0.9, 1.4, 1.5}, kTwo[] = {1.3, 1.9, 2.3};
    const int64_t w = wgs(128) * n;
    if (w - wgs(128) < 1024) offer(ROWS_TILES, n, rounds(w, 512) * (steps + 4) * (w <= 256 ? kOne[dim] : kTwo[dim]) + join_us(n));
    // 256 rows, one on a CU (2048 rows x 16 heads of 72 over 2048 keys: 44 us against 59)
    constexpr double kWide[] = {1.0, 1.2, 1.7};
    if (dt == DT_BF16 && wgs(256) * (n - 1) < 512) offer(ROWS_WIDE, n, rounds(wgs(256) * n, 256) * (steps * kWide[dim] + 8) + join_us(n));
  }

  // The key kernel for single tokens, and for launches that leave the chip empty.  It reads the keys for every 32 rows, through the
  // L2s at some 8 TB/s (1024 rows x 16 heads of 72 over 1024 keys: 18 us, in tiles 30; 512 rows x 8 heads of 128 over 16384
  // keys: 188 and 63).  In fp32 the matrix units bound all kernels, and more waves are better until the chip holds them (1024
  // rows x 16 heads of 128 over as many keys: 88 us, in tiles 121).
  const double keys_us = 4.0 + (double)wgs(32) * max_kv * head_dim * 2 * dt_size(dt) / 8e6;
  if (rows <= (int64_t)n_seqs * 32 || (dt == DT_BF16 ? keys_us < best : wgs(32) <= 1024)) {
    // Chunks down to 256 keys while there is no more than a workgroup for every CU (one token of 8 key heads over 4096 keys: 16 chunks
    // 13.5 us, 4 chunks 21.3; of 2 key heads over 131072 keys: 128 chunks 30.6 us, 64 chunks 34.0, 256 chunks 33.0; 20 tokens of 8
    // over 4096: whole 54, in two chunks 66).  Behind that, chunks of at least 2048 keys, whole rounds of the 512
    // workgroups that the chip holds, up to 8192: caches of different lengths share the chip evenly (64 tokens over up to 16384 keys of
    // 8 key heads: 150 us, without chunks 211, with chunks of 1024 keys 177; where lengths are alike it costs little: 32 tokens
    // over 8192 keys each 176, in two chunks 173).
    const int64_t w = wgs(32), none = 1;
    int64_t n = std::min(std::max(256 / w, none), std::max(max_kv / 256, none));
    int64_t more = std::min((8192 + w - 1) / w, max_kv / 2048);
    if (w < 512) more -= more % (512 / w);
    n = std::max(n, more);
    p = RowsPlan{ROWS_KEYS, (int)(n < kMaxChunks ? n : kMaxChunks), n == more ? 2048 : 256, 0};
  }
  if (p.splits > 1) p.ws_bytes = (size_t)p.splits * total_q * n_heads * (head_dim + 2) * sizeof(float);
  return p;
}

hipError_t launch_rows_join(const RowsAttn &a, hipStream_t s) { return a.dt == DT_BF16 ? launch_join<bf16_t>(a, s) : launch_join<float>(a, s); }

hipError_t launch_rows_attention(const RowsAttn &a, hipStream_t s) {
  return a.dt == DT_BF16 ? launch_type<bf16_t>(a, s) : launch_type<float>(a, s);
}

}  // namespace pf
