// Norm and rotation of the heads of packed rows, the same with the write of keys and values into pages of 8- or 4-bit numbers, and these
// pages read back.
//
// A head is normed over its channels, y = (x - mean) r w + b, and turned, z_c = y_c C_c + y_partner(c) S_c with the cosine of the channel's pair and
// its sine, minus for the pair's first channel.  Angles as in rope_rows.hip: turns in 64 bits up to the fraction.  A block of 32 channels of a
// key or value then becomes codes of x / 2^e, e the least exponent under which its largest magnitude fits.
//
// Bound by memory: a row is read once and written once.  A head is spread over as many lanes as it has units of 16 bytes, a wave takes as
// many heads as that leaves room for, so the sums over a head and the largest of a block are exchanges within the wave.
#include <algorithm>

#include "mx.h"
#include "requests.h"

namespace pf {
namespace {

constexpr int kMaxPairs = PF_ROPE_MAX_PAIRS, kMaxDim = 128, kWaves = 4, kMaxTok = 8;
constexpr int V = 8;                                 // channels of a lane's unit
enum { TURN_PAIRS, TURN_HALVES, TURN_HALVES_ANY };   // neighbours; an axis' half apart, the halves whole units or not

struct TurnK {
  double turns[kMaxPairs];
  float magnitude;
  int n_axes, rot;                  // rot: channels that turn
  int axis_end[PF_ROPE_MAX_AXES];   // running end of the axes, in pairs
};

struct HeadsK {
  HeadRows r;
  int tok;               // tokens of a workgroup
  int t0;                // first token of the launch
};

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

// A choice between values: `c ? a : b` of two arguments of a kernel is one of their addresses, from which lanes then load.
template <typename T>
__device__ __forceinline__ T pick(bool c, T a, T b) { return c ? a : b; }

// V channels of a row as they are in memory.
template <typename T>
struct Unit {
  static constexpr int N = V * (int)sizeof(T) / 16;
  u32x4 w[N];
  __device__ __forceinline__ void load(const T *p, bool once) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const u32x4 *from = reinterpret_cast<const u32x4 *>(p) + i;
      w[i] = once ? __builtin_nontemporal_load(from) : *from;
    }
  }
  __device__ __forceinline__ void store(T *p) const {
#pragma unroll
    for (int i = 0; i < N; ++i) reinterpret_cast<u32x4 *>(p)[i] = w[i];
  }
  __device__ __forceinline__ float operator[](int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i / 4][i % 4]);
    else return __uint_as_float(i & 1 ? w[0][i / 2] & 0xffff0000u : w[0][i / 2] << 16);
  }
  __device__ __forceinline__ void round(const float (&x)[V]) {
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      if constexpr (sizeof(T) == 4) {
        w[i / 4][i % 4] = __float_as_uint(x[i]);
        w[i / 4][i % 4 + 1] = __float_as_uint(x[i + 1]);
      } else {
        w[0][i / 2] = (unsigned)__builtin_bit_cast(unsigned short, (bf16_t)x[i]) | (unsigned)__builtin_bit_cast(unsigned short, (bf16_t)x[i + 1]) << 16;
      }
    }
  }
};

#if defined(__HIP_DEVICE_COMPILE__)
template <int CTRL>
__device__ __forceinline__ unsigned across(unsigned v) { return (unsigned)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xf, 0xf, true); }
#else   // the host pass only parses the kernels
template <int CTRL>
__device__ unsigned across(unsigned v) { return v; }
#endif
constexpr int kSwap1 = 0xb1, kSwap2 = 0x4e, kMirror8 = 0x141, kMirror16 = 0x140;   // lanes ^ 1, ^ 2, and 8 or 16 lanes back to front

// A head's n lanes (at most 16), lane - u the first of them.  N = n of 8 or 16: they do not cross a row of 16 lanes, within which lanes exchange
// values without LDS; 0: any n.  Lanes that belong to no head take part with what they have.
template <int N>
struct HeadLanes {
  int lane, u, n;
  __device__ __forceinline__ float sum(float v) const {
    if constexpr (N != 0) {
      v += __uint_as_float(across<kSwap1>(__float_as_uint(v)));
      v += __uint_as_float(across<kSwap2>(__float_as_uint(v)));
      v += __uint_as_float(across<kMirror8>(__float_as_uint(v)));
      if constexpr (N == 16) v += __uint_as_float(across<kMirror16>(__float_as_uint(v)));
      return v;
    }
#pragma unroll
    for (int o = 8; o > 0; o /= 2)
      if (o < n) {
        const float y = __shfl(v, lane + o, kWave);
        if (u < o && u + o < n) v += y;
      }
    return __shfl(v, lane - u, kWave);
  }
  // The largest of the block of four lanes (the last one of a head may be shorter).
  __device__ __forceinline__ unsigned block_max(unsigned v) const {
    static_assert(PF_MX_BLOCK == 4 * V, "a block is four lanes");
    if constexpr (N != 0) {
      v = max(v, across<kSwap1>(v));
      return max(v, across<kSwap2>(v));
    }
#pragma unroll
    for (int o = 1; o < 4; o *= 2) {
      const int to = u ^ o;
      v = max(v, (unsigned)__shfl((int)v, lane - u + (to < n ? to : u), kWave));
    }
    return v;
  }
};

// 1 / sqrt(x): the hardware's, within a unit; for fp32 rows with a step of Newton's behind it.  Tiny sums are scaled, it takes no subnormal ones.
template <typename T>
__device__ __forceinline__ float inverse_root(float x) {
  const bool tiny = x < 0x1p-100f;
  const float y = tiny ? x * 0x1p100f : x;
  float r = __builtin_amdgcn_rsqf(y);
  if constexpr (sizeof(T) == 4) {
    const float better = fmaf(0.5f * r, fmaf(-y * r, r, 1.0f), r);
    r = r == 0.f || y == 0.f ? r : better;
  }
  return tiny ? r * 0x1p50f : r;
}

// Codes of the V values of a block whose largest magnitude has the bits `most`, and the exponent's byte.
template <int FMT>
__device__ __forceinline__ unsigned encode(const float (&x)[V], unsigned most, unsigned (&code)[V * Mx<FMT>::BITS / 32]) {
  using M = Mx<FMT>;
  constexpr unsigned top_mant = M::kTop & 0x7fffffu;
  const int e = clampi((int)((most + 0x7fffffu - top_mant) >> 23) - (int)(M::kTop >> 23), M::kLeast, M::kMost);
  const float down = __uint_as_float((unsigned)(127 - e) << 23);   // a power of two: the product is exact
  const float top = __uint_as_float(M::kTop);
  const bool none = most >= 0x7f800000u;
  float y[V];
#pragma unroll
  for (int i = 0; i < V; ++i) y[i] = __builtin_amdgcn_fmed3f(x[i] * down, -top, top);
#pragma unroll
  for (unsigned &w : code) w = 0;
#if defined(__HIP_DEVICE_COMPILE__)
  if constexpr (FMT == PF_MX_E4M3) {
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      code[i / 4] = __builtin_amdgcn_cvt_pk_fp8_f32(y[i], y[i + 1], code[i / 4], false);
      code[i / 4] = __builtin_amdgcn_cvt_pk_fp8_f32(y[i + 2], y[i + 3], code[i / 4], true);
    }
  } else {
    code[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code[0], y[0], y[1], 1.0f, 0);
    code[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code[0], y[2], y[3], 1.0f, 1);
    code[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code[0], y[4], y[5], 1.0f, 2);
    code[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code[0], y[6], y[7], 1.0f, 3);
  }
#endif
#pragma unroll
  for (unsigned &w : code) w = none ? 0 : w;
  return none ? 255u : (unsigned)(e + 127);
}

// A lane's heads, step after step: `fit` heads to a wave at a step, the workgroup's tokens behind each other with `heads` heads each, from
// the wave's place on and `stride` heads further each time.
struct Walk {
  int heads, steps, stride, stride_t, stride_h;
  struct At {
    int at, t, h;        // place, token, head
  };
  __device__ __forceinline__ Walk(int heads_, int tok, int fit) : heads(heads_), steps(tok * heads_), stride(gridDim.y * kWaves * fit) {
    stride_t = stride / heads;
    stride_h = stride - stride_t * heads;
  }
  __device__ __forceinline__ At first(int wave, int fit, int sub) const {
    const int at = (blockIdx.y * kWaves + wave) * fit + sub;
    return At{at, at / heads, at % heads};
  }
  __device__ __forceinline__ void next(At &w) const {
    w.at += stride;
    w.t += stride_t;
    w.h += stride_h;
    if (w.h >= heads) {
      w.h -= heads;
      ++w.t;
    }
  }
};

// Where packed row `row` of a call goes in the pages: page (-1: none, -2: the row belongs to no sequence) and row of the page.
__device__ __forceinline__ void find_slot(const Pages &pages, const int32_t *cu, const int32_t *first, int n_seqs, int row, int lane, int64_t &page, int &in_page) {
  page = -2;
  in_page = 0;
  const int s = wave_search(n_seqs, lane, row, [&](int i) { return cu[i]; });
  if (s < 0 || s >= n_seqs) return;
  page = -1;
  const int64_t slot = (int64_t)first[s] + ((int64_t)row - cu[s]);
  if (slot < 0 || slot >= ((int64_t)pages.max_pages << pages.page_shift)) return;
  const int pg = pages.table[(int64_t)s * pages.max_pages + (slot >> pages.page_shift)];
  if (pg < 0 || pg >= pages.n_pages) return;
  page = pg;
  in_page = (int)(slot & ((1 << pages.page_shift) - 1));
}

// FMT < 0: q and k rows to rows; else k and v into pages.  LAYOUT: of the pairs.  N: lanes of a head (0: any number).  A workgroup takes tok tokens, a wave `fit` heads at a
// step and kDepth steps' loads at a time, the first of them before the tables are worked out.
template <typename T> constexpr int kDepth = sizeof(T) == 2 ? 2 : 1;
template <typename T, int FMT, int LAYOUT, int N>
__global__ __launch_bounds__(64 * kWaves) void head_rows_kernel(TurnK rk, HeadsK p) {
#pragma clang fp contract(off)   // the same rows from all instances: pages get what pf_op_qk_norm_rope gives
  constexpr bool APPEND = FMT >= 0, HALF = LAYOUT != TURN_PAIRS;
  constexpr int DEPTH = kDepth<T>;
  const HeadRows &a = p.r;
  __shared__ __attribute__((aligned(16))) float cosine[kMaxTok][kMaxDim], sine[kMaxTok][kMaxDim];
  __shared__ __attribute__((aligned(16))) float other[HALF ? kWaves : 1][HALF ? 64 * V : 1];   // the wave's units, for the pairs' other channels
  // of a token: bytes from the pages' start to its row of head 0 of k and v, and to its exponents; -1: no page, -2: the row belongs to no sequence
  __shared__ int64_t code_at[kMaxTok][2], exp_at[kMaxTok][2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int t0 = p.t0 + blockIdx.x * p.tok, dh = N ? N * V : a.head_dim, pairs = rk.rot >> 1;
  const int tokens = a.tokens - t0;                         // of this workgroup and behind it

  const int n = N ? N : dh / V, fit = 64 / n;               // lanes of a head, heads of a wave
  const int sub = lane / n, u = lane - sub * n, c0 = u * V; // the lane's head of these, unit and first channel
  const HeadLanes<N> head{lane, u, n};
  const int n_heads = a.n_heads, from_v = APPEND ? a.n_heads + a.kv_heads : 1 << 30;
  const Walk walk(a.n_heads + (APPEND ? 2 : 1) * a.kv_heads, p.tok, fit);
  Walk::At now = walk.first(wave, fit, sub);
  // rows of the workgroup's first token, and elements from there: with more than one token to a workgroup the launch keeps them inside 32 bits
  const T *const q = (const T *)a.q + t0 * a.ldq, *const k = (const T *)a.k + t0 * a.ldk, *const v = (const T *)a.v + t0 * a.ldv;
  T *const q_out = (T *)a.q_out + t0 * a.ldqo, *const k_out = (T *)a.k_out + t0 * a.ldko;
  const int ldq = (int)a.ldq, ldk = (int)a.ldk, ldv = (int)a.ldv, ldqo = (int)a.ldqo, ldko = (int)a.ldko;
  const auto there = [&](const Walk::At &w) __attribute__((always_inline)) { return sub < fit && w.at < walk.steps && w.t < tokens; };
  Unit<T> raw[DEPTH];
  const auto load = [&](Walk::At w) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < DEPTH; ++j, walk.next(w)) {
      const bool is_q = w.h < n_heads, is_v = w.h >= from_v;
      const T *src = pick(is_q, q, pick(is_v, v, k));
      const int h = w.h - pick(is_q, 0, pick(is_v, from_v, n_heads)), ld = pick(is_q, ldq, pick(is_v, ldv, ldk));
#pragma unroll
      for (int i = 0; i < Unit<T>::N; ++i) raw[j].w[i] = u32x4{0, 0, 0, 0};
      if (there(w)) raw[j].load(src + (w.t * ld + h * dh + c0), a.once);
    }
  };
  load(now);

  // the norms' vectors, the lane's channels of them
  const bool norms = a.norm[0].kind != PF_NORM_NONE || a.norm[1].kind != PF_NORM_NONE;
  const bool layer = a.norm[0].kind == PF_NORM_LAYER || a.norm[1].kind == PF_NORM_LAYER;
  const bool biased = a.norm[0].bias || a.norm[1].bias;
  Unit<T> weight[2], bias[2];
  if (norms) {
    float one[V], none[V];
#pragma unroll
    for (int i = 0; i < V; ++i) one[i] = 1.f, none[i] = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      weight[i].round(one);
      bias[i].round(none);
      if (a.norm[i].weight) weight[i].load((const T *)a.norm[i].weight + c0, false);
      if (a.norm[i].bias) bias[i].load((const T *)a.norm[i].bias + c0, false);
    }
  }

  // cosines and sines of the workgroup's tokens by channel
  for (int e = tid; e < p.tok * pairs; e += 64 * kWaves) {
    const int t = e / pairs, i = e - t * pairs;
    if (t >= tokens) break;
    const int end0 = rk.axis_end[0], end1 = rk.axis_end[1];
    const int axis = (i >= end0) + (rk.n_axes > 1 && i >= end1);
    const double turns = (double)a.pos[(int64_t)(t0 + t) * rk.n_axes + axis] * rk.turns[i];
    float sn, c;
    sincospif(2.0f * (float)(turns - rint(turns)), &sn, &c);
    const int from = pick(axis == 0, 0, pick(axis == 1, end0, end1)), w = pick(axis == 0, end0, pick(axis == 1, end1, rk.axis_end[2])) - from;
    const int one = HALF ? 2 * from + (i - from) : 2 * i, two = HALF ? one + w : one + 1;
    cosine[t][one] = cosine[t][two] = c * rk.magnitude;
    sine[t][one] = -sn * rk.magnitude;
    sine[t][two] = sn * rk.magnitude;
  }
  if constexpr (APPEND) {
    for (int t = wave; t < p.tok; t += kWaves) {
      int64_t page = -2;
      int row = 0;
      if (t < tokens) find_slot(a.pages, a.cu, a.first, a.n_seqs, t0 + t, lane, page, row);
      if (lane == 0) {
        code_at[t][0] = page < 0 ? page : page * a.pages.k_stride + row * a.mx.row_bytes;
        code_at[t][1] = page < 0 ? page : page * a.pages.v_stride + row * a.mx.row_bytes;
        exp_at[t][0] = page * a.mx.k_scale_stride + row * a.mx.blocks;
        exp_at[t][1] = page * a.mx.v_scale_stride + row * a.mx.blocks;
      }
    }
  }
  __syncthreads();

  const float inv = 1.0f / (float)dh;
  const int kind_q = a.norm[0].kind, kind_k = a.norm[1].kind;
  const float eps_q = a.norm[0].eps, eps_k = a.norm[1].eps;
  // where the pairs' other channels are, from the lane's own
  int to[LAYOUT == TURN_HALVES_ANY ? V : 1];
  if constexpr (HALF) {
#pragma unroll
    for (int i = 0; i < (LAYOUT == TURN_HALVES_ANY ? V : 1); ++i) {
      const int c = c0 + i, e0 = 2 * rk.axis_end[0], e1 = rk.n_axes > 1 ? 2 * rk.axis_end[1] : rk.rot;
      const int from = c < e0 ? 0 : c < e1 ? e0 : e1, end = c < e0 ? e0 : c < e1 ? e1 : rk.rot, w = (end - from) >> 1;
      to[i] = c >= rk.rot ? 0 : c < from + w ? w : -w;
    }
  }

  const auto work = [&](const Walk::At &w, Unit<T> &unit) __attribute__((always_inline)) {
    const bool is_q = w.h < n_heads, is_v = w.h >= from_v;
    const int h = w.h - pick(is_q, 0, pick(is_v, from_v, n_heads));
    const int t = min(w.t, kMaxTok - 1);
    bool live = there(w);
    int64_t at = 0;
    if constexpr (APPEND) {   // rows that belong to no sequence stay as they are, in q_out too
      at = code_at[t][is_v];
      live = live && at >= (is_q ? -1 : 0);
    }
    float x[V];
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = unit[i];
    if (norms) {
      const int kind = pick(is_v, (int)PF_NORM_NONE, pick(is_q, kind_q, kind_k));
      if (layer) {
        float t1 = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) t1 += x[i];
        float mean = head.sum(t1) * inv;
        mean = kind == PF_NORM_LAYER ? mean : 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] -= mean;
      }
      float t2 = 0.f;
#pragma unroll
      for (int i = 0; i < V; ++i) t2 = fmaf(x[i], x[i], t2);
      float r = inverse_root<T>(fmaf(head.sum(t2), inv, pick(is_q, eps_q, eps_k)));
      r = kind == PF_NORM_NONE ? 1.f : r;
      Unit<T> g;
#pragma unroll
      for (int i = 0; i < Unit<T>::N; ++i) g.w[i] = pick(is_q, weight[0].w[i], weight[1].w[i]);
#pragma unroll
      for (int i = 0; i < V; ++i) x[i] = x[i] * r * (is_v ? 1.f : g[i]);
      if (biased) {
#pragma unroll
        for (int i = 0; i < Unit<T>::N; ++i) g.w[i] = pick(is_q, bias[0].w[i], bias[1].w[i]);
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] += is_v ? 0.f : g[i];
      }
    }
    if (rk.rot) {
      float y[V], cs[V], sn[V];
      if constexpr (HALF) {
        float *mine = other[wave] + min(sub * dh + c0, 63 * V);
#pragma unroll
        for (int i = 0; i < V; i += 4) *reinterpret_cast<float4 *>(mine + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
        __builtin_amdgcn_wave_barrier();
        if constexpr (LAYOUT == TURN_HALVES) {
#pragma unroll
          for (int i = 0; i < V; i += 4) {
            const float4 z = *reinterpret_cast<const float4 *>(mine + to[0] + i);
            y[i] = z.x, y[i + 1] = z.y, y[i + 2] = z.z, y[i + 3] = z.w;
          }
        } else {
#pragma unroll
          for (int i = 0; i < V; ++i) y[i] = mine[i + to[i]];
        }
        __builtin_amdgcn_wave_barrier();
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = x[i ^ 1];
      }
#pragma unroll
      for (int i = 0; i < V; i += 4) {
        const float4 z = *reinterpret_cast<const float4 *>(&cosine[t][c0 + i]), s = *reinterpret_cast<const float4 *>(&sine[t][c0 + i]);
        cs[i] = z.x, cs[i + 1] = z.y, cs[i + 2] = z.z, cs[i + 3] = z.w;
        sn[i] = s.x, sn[i + 1] = s.y, sn[i + 2] = s.z, sn[i + 3] = s.w;
      }
      const int end = is_v ? 0 : rk.rot;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float z = fmaf(x[i], cs[i], y[i] * sn[i]);
        x[i] = c0 + i < end ? z : x[i];
      }
    }
    // rounded to the rows' type, which is what the pages get too
    unit.round(x);
    if (live && (!APPEND || is_q)) unit.store(pick(is_q, q_out, k_out) + (w.t * pick(is_q, ldqo, ldko) + h * dh + c0));
    if constexpr (APPEND) {
      unsigned most = 0;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        x[i] = unit[i];
        most = max(most, __float_as_uint(x[i]) & 0x7fffffffu);
      }
      most = head.block_max(most);
      constexpr int BYTES = V * Mx<FMT>::BITS / 8;
      unsigned code[BYTES / 4];
      const unsigned byte = encode<FMT>(x, most, code);
      if (!is_q && live) {
        const int64_t rows = (int64_t)h << a.pages.page_shift;
        uint8_t *to_row = pick(is_v, (uint8_t *)a.pages.v, (uint8_t *)a.pages.k) + (at + rows * a.mx.row_bytes);
        if constexpr (BYTES == 8) *reinterpret_cast<u32x2 *>(to_row + u * BYTES) = u32x2{code[0], code[1]};
        else *reinterpret_cast<unsigned *>(to_row + u * BYTES) = code[0];
        if (u % 4 == 0) pick(is_v, a.mx.v_scale, a.mx.k_scale)[exp_at[t][is_v] + rows * a.mx.blocks + u / 4] = (uint8_t)byte;
        if (u == n - 1)   // zeros up to whole 16 bytes: words, as head_dim is a multiple of 8
          for (int b = n * BYTES; b < a.mx.row_bytes; b += 4) *reinterpret_cast<unsigned *>(to_row + b) = 0;
      }
    }
  };
  for (;;) {
#pragma unroll
    for (int j = 0; j < DEPTH; ++j, walk.next(now)) {
      if (__builtin_amdgcn_readfirstlane(now.at - sub) >= walk.steps) return;
      work(now, raw[j]);
    }
    load(now);
  }
}

// Slots of pages to rows: a workgroup takes tok tokens, a wave `fit` heads at a step and READ_DEPTH steps' loads at a time.
struct ReadK {
  MxRead r;
  int tok, t0;
};
constexpr int kMaxReadTok = 32, READ_DEPTH = 4;
template <typename T, int FMT>
__global__ __launch_bounds__(64 * kWaves) void mx_read_kernel(ReadK p) {
  constexpr int BYTES = V * Mx<FMT>::BITS / 8;
  const MxRead &a = p.r;
  __shared__ int64_t page_of[kMaxReadTok];
  __shared__ int row_of[kMaxReadTok];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int t0 = p.t0 + blockIdx.x * p.tok, dh = a.head_dim;
  for (int t = wave; t < p.tok; t += kWaves) {
    int64_t page = -2;
    int in_page = 0;
    if (t0 + t < a.tokens) find_slot(a.pages, a.cu, a.first, a.n_seqs, t0 + t, lane, page, in_page);
    if (lane == 0) {
      page_of[t] = page;
      row_of[t] = in_page;
    }
  }
  __syncthreads();
  const int n = dh / V, fit = 64 / n, sub = lane / n, u = lane - sub * n;
  const int sides = (a.k_out != nullptr) + (a.v_out != nullptr);
  const Walk walk(sides * a.kv_heads, p.tok, fit);
  Walk::At now = walk.first(wave, fit, sub);
  while (__builtin_amdgcn_readfirstlane(now.at - sub) < walk.steps) {
    unsigned code[READ_DEPTH][2];
    unsigned exp[READ_DEPTH];
    T *to[READ_DEPTH];
#pragma unroll
    for (int j = 0; j < READ_DEPTH; ++j, walk.next(now)) {
      code[j][0] = code[j][1] = exp[j] = 0;
      to[j] = nullptr;
      if (sub >= fit || now.at >= walk.steps) continue;
      const int64_t page = page_of[now.t];
      if (page < -1) continue;
      const bool is_v = !a.k_out || now.h >= a.kv_heads;
      const int h = is_v && a.k_out ? now.h - a.kv_heads : now.h;
      to[j] = pick(is_v, (T *)a.v_out, (T *)a.k_out) + ((t0 + now.t) * pick(is_v, a.ldv, a.ldk) + h * dh + u * V);
      if (page < 0) continue;
      const int64_t in_page = ((int64_t)h << a.pages.page_shift) + row_of[now.t];
      const uint8_t *from = pick(is_v, (const uint8_t *)a.pages.v, (const uint8_t *)a.pages.k) + (page * pick(is_v, a.pages.v_stride, a.pages.k_stride) + in_page * a.mx.row_bytes + u * BYTES);
      exp[j] = pick(is_v, a.mx.v_scale, a.mx.k_scale)[page * pick(is_v, a.mx.v_scale_stride, a.mx.k_scale_stride) + in_page * a.mx.blocks + u / 4];
      if constexpr (BYTES == 8) {
        const u32x2 x = *reinterpret_cast<const u32x2 *>(from);
        code[j][0] = x[0], code[j][1] = x[1];
      } else {
        code[j][0] = *reinterpret_cast<const unsigned *>(from);
      }
    }
#pragma unroll
    for (int j = 0; j < READ_DEPTH; ++j) {
      Unit<T> out;
      mx_unit<FMT>(code[j], mx_power(exp[j]), out.w);
      if (to[j]) out.store(to[j]);
    }
  }
}

// Workgroups along y for launches of few tokens: a token's `parts` turns of a workgroup are split over them while they are few.
int split(int tokens, int parts) {
  int y = std::max(parts, 1);
  while (y > 1 && (int64_t)tokens * y > 4096) y = (y + 1) / 2;
  return y;
}

template <typename T, int FMT, int LAYOUT, int N>
hipError_t launch_heads(const TurnK &rk, HeadsK p, hipStream_t s) {
  const int per_turn = 64 / (p.r.head_dim / V) * kWaves, heads = p.r.n_heads + (FMT >= 0 ? 2 : 1) * p.r.kv_heads;
  const int64_t ld = std::max(std::max(std::max(p.r.ldq, p.r.ldqo), std::max(p.r.ldk, p.r.ldko)), p.r.ldv);
  p.tok = p.r.tokens < 4096 || ld > INT32_MAX / kMaxTok / 2 ? 1 : std::min(std::max(kDepth<T> * per_turn / heads, 1), kMaxTok);
  const int y = p.tok == 1 ? split(p.r.tokens, (heads + per_turn - 1) / per_turn) : 1;
  hipError_t e = hipSuccess;
  for (p.t0 = 0; p.t0 < p.r.tokens && e == hipSuccess; p.t0 += kLaunchRows) {
    const int rows = std::min(p.r.tokens - p.t0, kLaunchRows);
    head_rows_kernel<T, FMT, LAYOUT, N><<<dim3((rows + p.tok - 1) / p.tok, y), 64 * kWaves, 0, s>>>(rk, p);
    e = hipGetLastError();
  }
  return e;
}

template <typename T, int FMT, int LAYOUT>
hipError_t launch_lanes(const TurnK &rk, const HeadsK &p, hipStream_t s) {
  if (p.r.head_dim == 128) return launch_heads<T, FMT, LAYOUT, 16>(rk, p, s);
  if (p.r.head_dim == 64) return launch_heads<T, FMT, LAYOUT, 8>(rk, p, s);
  return launch_heads<T, FMT, LAYOUT, 0>(rk, p, s);
}
template <typename T, int FMT>
hipError_t launch_layout(const TurnK &rk, const HeadsK &p, bool half, int align, hipStream_t s) {
  if (half && align % V) return launch_heads<T, FMT, TURN_HALVES_ANY, 0>(rk, p, s);
  return half ? launch_lanes<T, FMT, TURN_HALVES>(rk, p, s) : launch_lanes<T, FMT, TURN_PAIRS>(rk, p, s);
}
template <typename T>
hipError_t launch_format(const TurnK &rk, const HeadsK &p, bool half, int align, hipStream_t s) {
  if (!p.r.n_seqs) return launch_layout<T, -1>(rk, p, half, align, s);
  return p.r.mx.format == PF_MX_E4M3 ? launch_layout<T, PF_MX_E4M3>(rk, p, half, align, s) : launch_layout<T, PF_MX_E2M1>(rk, p, half, align, s);
}

template <typename T, int FMT>
hipError_t launch_read(ReadK p, hipStream_t s) {
  const int per_turn = 64 / (p.r.head_dim / V) * kWaves, heads = ((p.r.k_out != nullptr) + (p.r.v_out != nullptr)) * p.r.kv_heads;
  p.tok = p.r.tokens < 4096 ? 1 : std::min(std::max(READ_DEPTH * per_turn / heads, 1), kMaxReadTok);
  const int y = p.tok == 1 ? split(p.r.tokens, (heads + per_turn - 1) / per_turn) : 1;
  hipError_t e = hipSuccess;
  for (p.t0 = 0; p.t0 < p.r.tokens && e == hipSuccess; p.t0 += kLaunchRows) {
    const int rows = std::min(p.r.tokens - p.t0, kLaunchRows);
    mx_read_kernel<T, FMT><<<dim3((rows + p.tok - 1) / p.tok, y), 64 * kWaves, 0, s>>>(p);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

hipError_t launch_head_rows(const HeadRows &args, const pf_rope *rope, hipStream_t s) {
  if (args.tokens <= 0) return hipSuccess;
  TurnK rk{};
  bool half = false;
  int align = 0;   // greatest power of two that divides every axis' half width, and the places where the axes start
  if (rope) {
    rk.magnitude = rope->magnitude;
    rk.n_axes = rope->n_axes;
    int end = 0;
    for (int i = 0; i < rope->n_axes; ++i) {
      end += rope->axis_dim[i] / 2;
      rk.axis_end[i] = end;
      align |= rope->axis_dim[i] / 2;
    }
    align &= -align;
    rk.rot = 2 * end;
    for (int i = 0; i < end; ++i) rk.turns[i] = rope->turns[i];
    half = rope->layout == PF_ROPE_HALF;
  }
  HeadsK p{args, 1, 0};
  p.r.once = (int64_t)args.tokens * 2 * (args.n_heads + 2 * args.kv_heads) * args.head_dim * (int64_t)dt_size(args.dt) > kReadOnceBytes;
  return args.dt == DT_BF16 ? launch_format<bf16_t>(rk, p, half, align, s) : launch_format<float>(rk, p, half, align, s);
}

hipError_t launch_mx_read(const MxRead &r, hipStream_t s) {
  if (r.tokens <= 0) return hipSuccess;
  const ReadK p{r, 1, 0};
  if (r.dt == DT_BF16) return r.mx.format == PF_MX_E4M3 ? launch_read<bf16_t, PF_MX_E4M3>(p, s) : launch_read<bf16_t, PF_MX_E2M1>(p, s);
  return r.mx.format == PF_MX_E4M3 ? launch_read<float, PF_MX_E4M3>(p, s) : launch_read<float, PF_MX_E2M1>(p, s);
}

}  // namespace pf
