// Rotary positions on packed rows, and the same with the write of keys and values into pages.
//
// Pair i of an axis of width w turns by pos * theta^(-2i/w), its frequency stretched or not (pf_rope_init):
// (a, b) -> m (a cos - b sin, a sin + b cos).  An angle is kept as a number of turns in 64 bits, pos * f / 2 pi, and only
// its fraction goes on in 32 bits: at position 10^6 a 32-bit angle would already be off by 0.03 rad.  A fraction, sine and cosine of 24 bits are
// within a rounding or two of the rows' own (fp32 rows: 5.3e-8 from the 64-bit result in the mean, with them in 64 bits 4.2e-8).
//
// Bound by memory (a row is read once and written once).  A workgroup takes one or a few tokens; it works out the
// (cos, sin) of their pairs once, into LDS, and all heads of the token use them: one evaluation per token and pair, not per
// element.  Each thread then moves units of 16 bytes (of two such halves where the pairs lie half an axis apart).
// 16896 rows of 32 heads of 128, bf16, three axes: 46 us, 277 MB at 6.0 TB/s (a large device copy: 4.6; the end of what is written stays in the
// cache in front of the memory).  Append of 7178 fp32 rows of 3 x 16 heads of 72: 43 us, 198 MB at 4.6 TB/s.  48 or 128 rows: 3 - 4
// us, of launch and two memory latencies behind each other (position or sequence, then page; rows).
#include <algorithm>

#include "requests.h"

namespace pf {
namespace {

constexpr int kMaxPairs = PF_ROPE_MAX_PAIRS;

struct RopeK {
  double turns[kMaxPairs];
  float magnitude;
  int n_axes, rot;               // rot: channels that turn
  int axis_end[PF_ROPE_MAX_AXES];   // running end of the axes, in pairs
};

struct RowsK {
  const int32_t *pos;
  int tokens, head_dim;
  const void *q; int64_t ldq; void *q_out; int64_t ldqo; int n_heads;
  const void *k; int64_t ldk; const void *v; int64_t ldv; int kv_heads;
  Pages pages;
  const int32_t *cu, *first;
  int n_seqs;
  int t0;                // first token of the launch
};

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
template <typename T, int V> struct Unit { T e[V]; };
template <bool ONCE, typename T, int V> __device__ __forceinline__ void load_unit(const T *p, Unit<T, V> &u) {
  if constexpr (sizeof(T) * V == 16) {
    const u32x4 *from = reinterpret_cast<const u32x4 *>(p);
    *reinterpret_cast<u32x4 *>(&u) = ONCE ? __builtin_nontemporal_load(from) : *from;
  }
  else if constexpr (sizeof(T) * V == 8) *reinterpret_cast<uint2 *>(&u) = *reinterpret_cast<const uint2 *>(p);
  else u = *reinterpret_cast<const Unit<T, V> *>(p);
}
template <typename T, int V> __device__ __forceinline__ void store_unit(T *p, const Unit<T, V> &u) {
  if constexpr (sizeof(T) * V == 16) *reinterpret_cast<uint4 *>(p) = *reinterpret_cast<const uint4 *>(&u);
  else if constexpr (sizeof(T) * V == 8) *reinterpret_cast<uint2 *>(p) = *reinterpret_cast<const uint2 *>(&u);
  else *reinterpret_cast<Unit<T, V> *>(p) = u;
}

// HALF: pairs half an axis apart (each axis' half a multiple of V), else neighbours (V even).  TOK tokens per workgroup.
// ONCE: rows are read with non-temporal loads (units of 16 bytes).
template <typename T, int V, bool HALF, bool APPEND, int TOK, bool ONCE>
__global__ __launch_bounds__(256) void rope_rows_kernel(RopeK rk, RowsK a) {
  __shared__ float2 cs[TOK][kMaxPairs];
  __shared__ int64_t k_at[TOK], v_at[TOK];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int t0 = a.t0 + blockIdx.x * TOK;
  const int pairs = rk.rot >> 1, dh = a.head_dim;

  for (int e = tid; e < TOK * pairs; e += 256) {
    const int t = e / pairs, p = e - t * pairs;
    if (t0 + t >= a.tokens) break;
    const int axis = (p >= rk.axis_end[0]) + (rk.n_axes > 1 && p >= rk.axis_end[1]);
    const double turns = (double)a.pos[(int64_t)(t0 + t) * rk.n_axes + axis] * rk.turns[p];
    const float fr = (float)(turns - rint(turns));
    float sn, c;
    sincospif(2.0f * fr, &sn, &c);
    cs[t][p] = make_float2(c * rk.magnitude, sn * rk.magnitude);
  }
  if constexpr (APPEND) {
    for (int t = wave; t < TOK; t += 4) {
      int64_t ka = -1, va = -1;
      const int row = t0 + t;
      if (row < a.tokens) {
        const int s = wave_search(a.n_seqs, lane, row, [&](int i) { return a.cu[i]; });
        if (s >= 0 && s < a.n_seqs) {
          const int64_t slot = (int64_t)a.first[s] + ((int64_t)row - a.cu[s]);
          if (slot >= 0 && slot < ((int64_t)a.pages.max_pages << a.pages.page_shift)) {
            const int page = a.pages.table[(int64_t)s * a.pages.max_pages + (slot >> a.pages.page_shift)];
            if (page >= 0 && page < a.pages.n_pages) {
              const int64_t in_page = (slot & ((1 << a.pages.page_shift) - 1)) * dh;
              ka = page * a.pages.k_stride + in_page;
              va = page * a.pages.v_stride + in_page;
            }
          }
        }
      }
      if (lane == 0) {
        k_at[t] = ka;
        v_at[t] = va;
      }
    }
  }
  __syncthreads();

  // units of a turned head: HALF: `pairs / V` double units, then the channels behind them; else head_dim / V
  const int rot_units = HALF ? pairs / V : dh / V;
  const int head_units = HALF ? rot_units + (dh - rk.rot) / V : rot_units;
  const int copy_units = dh / V;
  const int turned = (a.n_heads + (APPEND ? a.kv_heads : 0)) * head_units;
  const int per_token = turned + (APPEND ? a.kv_heads * copy_units : 0);
  const int64_t head_stride = APPEND ? (int64_t)dh << a.pages.page_shift : 0;
  for (int e = blockIdx.y * 256 + tid; e < TOK * per_token; e += 256 * gridDim.y) {
    const int t = TOK == 1 ? 0 : e / per_token;
    const int u0 = e - t * per_token;
    const int64_t row = t0 + t;
    if (row >= a.tokens) break;
    const T *src;
    T *dst;
    int u;
    bool copy = false;
    if (u0 < turned) {
      const int h = u0 / head_units;
      u = u0 - h * head_units;
      if (h < a.n_heads) {
        src = (const T *)a.q + row * a.ldq + h * dh;
        dst = (T *)a.q_out + row * a.ldqo + h * dh;
        if constexpr (APPEND) {   // rows that belong to no sequence stay as they are, in q_out too
          if (row < a.cu[0] || row >= a.cu[a.n_seqs]) continue;
        }
      } else {
        if (k_at[t] < 0) continue;
        src = (const T *)a.k + row * a.ldk + (h - a.n_heads) * dh;
        dst = (T *)a.pages.k + k_at[t] + (h - a.n_heads) * head_stride;
      }
    } else {
      if (v_at[t] < 0) continue;
      const int h = (u0 - turned) / copy_units;
      u = u0 - turned - h * copy_units;
      src = (const T *)a.v + row * a.ldv + h * dh;
      dst = (T *)a.pages.v + v_at[t] + h * head_stride;
      copy = true;
    }
    if (copy || (HALF && u >= rot_units)) {
      const int c = copy ? u * V : rk.rot + (u - rot_units) * V;
      Unit<T, V> x;
      load_unit<ONCE>(src + c, x);
      store_unit(dst + c, x);
    } else if constexpr (HALF) {
      // pairs u * V .. + V - 1 lie in one axis: its first channel, and half its width
      const int p = u * V;
      const int b0 = 0, b1 = rk.axis_end[0], b2 = rk.n_axes > 1 ? rk.axis_end[1] : pairs;
      const int beg = p < b1 ? b0 : p < b2 ? b1 : b2;
      const int end = p < b1 ? b1 : p < b2 ? b2 : pairs;
      const int c = 2 * beg + (p - beg), hw = end - beg;
      Unit<T, V> x, y;
      load_unit<ONCE>(src + c, x);
      load_unit<ONCE>(src + c + hw, y);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float2 w = cs[t][p + i];
        const float xa = to_f32(x.e[i]), xb = to_f32(y.e[i]);
        x.e[i] = from_f32<T>(xa * w.x - xb * w.y);
        y.e[i] = from_f32<T>(xa * w.y + xb * w.x);
      }
      store_unit(dst + c, x);
      store_unit(dst + c + hw, y);
    } else {
      const int c = u * V;
      Unit<T, V> x;
      load_unit<ONCE>(src + c, x);
#pragma unroll
      for (int i = 0; i < V; i += 2) {
        if (c + i < rk.rot) {   // a unit may reach behind the channels that turn
          const float2 w = cs[t][(c + i) >> 1];
          const float xa = to_f32(x.e[i]), xb = to_f32(x.e[i + 1]);
          x.e[i] = from_f32<T>(xa * w.x - xb * w.y);
          x.e[i + 1] = from_f32<T>(xa * w.y + xb * w.x);
        }
      }
      store_unit(dst + c, x);
    }
  }
}

template <typename T, int V, bool HALF, bool APPEND, int TOK, bool ONCE>
hipError_t launch_parts(const RopeK &rk, RowsK a, int y, hipStream_t s) {
  static_assert(kLaunchRows % TOK == 0, "a launch ends with whole workgroups");
  hipError_t e = hipSuccess;
  for (a.t0 = 0; a.t0 < a.tokens && e == hipSuccess; a.t0 += kLaunchRows) {
    const int n = std::min(a.tokens - a.t0, kLaunchRows);
    rope_rows_kernel<T, V, HALF, APPEND, TOK, ONCE><<<dim3((n + TOK - 1) / TOK, y), 256, 0, s>>>(rk, a);
    e = hipGetLastError();
  }
  return e;
}

template <typename T, int V, bool HALF, bool APPEND, bool ONCE>
hipError_t launch_tok(const RopeK &rk, const RowsK &a, hipStream_t s) {
  // Workgroups of several tokens where a token has less than 256 threads' work and there are tokens for 2048 of them or more (4
  // tokens, 2, 1: 8192 tokens of 16 heads of 64, bf16, half layout, 64 units: 7.4, 8.3 and 9.0 us; append of 16384 of 16 + 2 x 16 heads
  // of 64, 256 units: 34.4, 33.1, 34.1; 16384 of 32 + 2 x 8 heads of 128, 448 units: 81, 79, 74).  A token's heads are split over
  // workgroups where there are few tokens.
  const int turned = HALF ? (rk.rot / 2 + a.head_dim - rk.rot) / V : a.head_dim / V;
  const int units = (a.n_heads + a.kv_heads) * turned + a.kv_heads * (a.head_dim / V);
  if (a.tokens >= 4096 && units <= 128) return launch_parts<T, V, HALF, APPEND, 4, ONCE>(rk, a, 1, s);
  if (a.tokens >= 4096 && units <= 256) return launch_parts<T, V, HALF, APPEND, 2, ONCE>(rk, a, 1, s);
  int y = (units + 255) / 256;
  while (y > 1 && (int64_t)a.tokens * y > 4096) y = (y + 1) / 2;
  return launch_parts<T, V, HALF, APPEND, 1, ONCE>(rk, a, y, s);
}

template <typename T, bool APPEND>
hipError_t launch_layout(const RopeK &rk, const RowsK &a, bool half, int align, hipStream_t s) {
  constexpr int V16 = 16 / (int)sizeof(T);
  const bool once = (int64_t)a.tokens * 2 * (a.n_heads + 2 * a.kv_heads) * a.head_dim * (int64_t)sizeof(T) > kReadOnceBytes;
  if (!half) return once ? launch_tok<T, V16, false, APPEND, true>(rk, a, s) : launch_tok<T, V16, false, APPEND, false>(rk, a, s);
  // pairs half an axis apart move in units that start on both halves' boundaries
  if (align % V16 == 0) return once ? launch_tok<T, V16, true, APPEND, true>(rk, a, s) : launch_tok<T, V16, true, APPEND, false>(rk, a, s);
  if (align % (V16 / 2) == 0) return launch_tok<T, V16 / 2, true, APPEND, false>(rk, a, s);
  return launch_tok<T, 1, true, APPEND, false>(rk, a, s);
}

}  // namespace

hipError_t launch_rope_rows(const RopeRows &r, hipStream_t s) {
  if (r.tokens <= 0) return hipSuccess;
  RopeK rk{};
  bool half = false;
  int align = 0;   // greatest power of two that divides every axis' half width
  if (r.rope) {
    const pf_rope &p = *r.rope;
    rk.magnitude = p.magnitude;
    rk.n_axes = p.n_axes;
    int end = 0;
    for (int i = 0; i < p.n_axes; ++i) {
      end += p.axis_dim[i] / 2;
      rk.axis_end[i] = end;
      align |= p.axis_dim[i] / 2;
    }
    align &= -align;
    rk.rot = 2 * end;
    for (int i = 0; i < end; ++i) rk.turns[i] = p.turns[i];
    half = p.layout == PF_ROPE_HALF;
  }
  RowsK a{r.pos, r.tokens, r.head_dim, r.q, r.ldq, r.q_out, r.ldqo, r.n_heads, r.k, r.ldk, r.v, r.ldv, r.n_seqs ? r.kv_heads : 0,
          r.pages, r.cu, r.first, r.n_seqs, 0};
  if (r.dt == DT_BF16)
    return r.n_seqs ? launch_layout<bf16_t, true>(rk, a, half, align, s) : launch_layout<bf16_t, false>(rk, a, half, align, s);
  return r.n_seqs ? launch_layout<float, true>(rk, a, half, align, s) : launch_layout<float, false>(rk, a, half, align, s);
}

}  // namespace pf
