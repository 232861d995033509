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

constexpr int kMaxPairs = PF_ROPE_MAX_PAIRS, kMaxDim = 128, kWaves = 4, kMaxTok = 4;
enum { TURN_PAIRS, TURN_HALVES, TURN_HALVES_ANY };   // neighbours; an axis' half apart, the halves whole units of 16 bytes or not

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

template <typename T>
__device__ __forceinline__ void widen(const u32x4 &raw, float (&x)[16 / sizeof(T)]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) {
      x[2 * i] = __uint_as_float(raw[i] << 16);
      x[2 * i + 1] = __uint_as_float(raw[i] & 0xffff0000u);
    } else {
      x[i] = __uint_as_float(raw[i]);
    }
  }
}

// A head's n lanes, lane - u the first of them.  Sums and maxima over all n, or over groups of `g` (a power of two) of them, the last
// one shorter; lanes that belong to no head take part with what they have.
struct HeadLanes {
  int lane, u, n;
  template <typename F>
  __device__ __forceinline__ float over(float v, F &&op) const {
    if ((n & (n - 1)) == 0) {
#pragma unroll
      for (int o = 1; o < 32; o *= 2)
        if (o < n) v = op(v, __shfl_xor(v, o, kWave));
      return v;
    }
#pragma unroll
    for (int o = 16; o > 0; o /= 2)
      if (o < n) {
        const float y = __shfl(v, lane + o, kWave);
        if (u < o && u + o < n) v = op(v, y);
      }
    return __shfl(v, lane - u, kWave);
  }
  __device__ __forceinline__ float sum(float v) const {
    return over(v, [](float a, float b) { return a + b; });
  }
  template <int G>
  __device__ __forceinline__ unsigned group_max(unsigned v) const {
#pragma unroll
    for (int o = 1; o < G; o *= 2) {
      const int to = u ^ o;
      v = max(v, (unsigned)__shfl((int)v, lane - u + (to < n ? to : u), kWave));
    }
    return v;
  }
};

// Codes of V values of a block whose largest magnitude has the bits `most`, and the exponent's byte.
template <int FMT, int V>
__device__ __forceinline__ unsigned encode(const float (&x)[V], unsigned most, unsigned (&code)[(V * Mx<FMT>::BITS + 31) / 32]) {
  using M = Mx<FMT>;
  constexpr unsigned top_mant = M::kTop & 0x7fffffu;
  const int e = clampi((int)((most + 0x7fffffu - top_mant) >> 23) - (int)(M::kTop >> 23), M::kLeast, M::kMost);
  const float down = __uint_as_float((unsigned)(127 - e) << 23);   // a power of two: the product is exact
  const float top = __uint_as_float(M::kTop);
  const bool none = most >= 0x7f800000u;
  float y[V];
#pragma unroll
  for (int i = 0; i < V; ++i) y[i] = fminf(fmaxf(x[i] * down, -top), top);
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
    if constexpr (V == 8) {
      code[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code[0], y[4], y[5], 1.0f, 2);
      code[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code[0], y[6], y[7], 1.0f, 3);
    }
  }
#endif
  if (none) {
#pragma unroll
    for (unsigned &w : code) w = 0;
  }
  return none ? 255u : (unsigned)(e + 127);
}

// FMT < 0: q and k rows to rows; else k and v into pages.  LAYOUT: of the pairs.
template <typename T, int FMT, int LAYOUT>
__global__ __launch_bounds__(64 * kWaves) void head_rows_kernel(TurnK rk, HeadsK p) {
#pragma clang fp contract(off)   // the same rows from all instances: pages get what pf_op_qk_norm_rope gives
  constexpr int V = 16 / (int)sizeof(T);
  constexpr bool APPEND = FMT >= 0, HALF = LAYOUT != TURN_PAIRS;
  const HeadRows &a = p.r;
  __shared__ __attribute__((aligned(16))) float cosine[kMaxTok][kMaxDim], sine[kMaxTok][kMaxDim];
  __shared__ __attribute__((aligned(16))) float other[HALF ? kWaves : 1][HALF ? 64 * V : 1];   // the wave's units, for the pairs' other channels
  __shared__ int64_t page_of[kMaxTok];      // -1: the row goes nowhere
  __shared__ int row_of[kMaxTok];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int t0 = p.t0 + blockIdx.x * p.tok, dh = a.head_dim, pairs = rk.rot >> 1;

  // cosines and sines of the workgroup's tokens by channel
  for (int e = tid; e < p.tok * pairs; e += 64 * kWaves) {
    const int t = e / pairs, i = e - t * pairs;
    if (t0 + t >= a.tokens) break;
    const int axis = (i >= rk.axis_end[0]) + (rk.n_axes > 1 && i >= rk.axis_end[1]);
    const double turns = (double)a.pos[(int64_t)(t0 + t) * rk.n_axes + axis] * rk.turns[i];
    float sn, c;
    sincospif(2.0f * (float)(turns - rint(turns)), &sn, &c);
    const int from = axis == 0 ? 0 : rk.axis_end[axis - 1], w = rk.axis_end[axis] - from;
    const int one = HALF ? 2 * from + (i - from) : 2 * i, two = HALF ? one + w : one + 1;
    cosine[t][one] = cosine[t][two] = c * rk.magnitude;
    sine[t][one] = -sn * rk.magnitude;
    sine[t][two] = sn * rk.magnitude;
  }
  if constexpr (APPEND) {
    for (int t = wave; t < p.tok; t += kWaves) {
      int64_t page = -1;
      int in_page = 0;
      const int row = t0 + t;
      if (row < a.tokens) {
        const int s = wave_search(a.n_seqs, lane, row, [&](int i) { return a.cu[i]; });
        if (s >= 0 && s < a.n_seqs) {
          const int64_t slot = (int64_t)a.first[s] + ((int64_t)row - a.cu[s]);
          if (slot >= 0 && slot < ((int64_t)a.pages.max_pages << a.pages.page_shift)) {
            const int pg = a.pages.table[(int64_t)s * a.pages.max_pages + (slot >> a.pages.page_shift)];
            if (pg >= 0 && pg < a.pages.n_pages) {
              page = pg;
              in_page = (int)(slot & ((1 << a.pages.page_shift) - 1));
            }
          }
        }
      }
      if (lane == 0) {
        page_of[t] = page;
        row_of[t] = in_page;
      }
    }
  }
  __syncthreads();

  const int n = dh / V, fit = 64 / n;                       // lanes of a head, heads of a wave
  const int sub = lane / n, u = lane - sub * n, c0 = u * V; // the lane's head of these, unit and first channel
  const HeadLanes head{lane, u, n};
  const int heads = a.n_heads + (APPEND ? 2 : 1) * a.kv_heads;
  const bool layer = a.norm[0].kind == PF_NORM_LAYER || a.norm[1].kind == PF_NORM_LAYER;
  const bool norms = a.norm[0].kind != PF_NORM_NONE || a.norm[1].kind != PF_NORM_NONE;
  // where the pairs' other channels are, from the lane's own
  int to[HALF ? V : 1];
  if constexpr (HALF) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = c0 + i, e0 = 2 * rk.axis_end[0], e1 = rk.n_axes > 1 ? 2 * rk.axis_end[1] : rk.rot;
      const int from = c < e0 ? 0 : c < e1 ? e0 : e1, end = c < e0 ? e0 : c < e1 ? e1 : rk.rot, w = (end - from) >> 1;
      to[i] = c >= rk.rot ? 0 : c < from + w ? w : -w;
    }
  }

  const int steps = p.tok * heads;
  for (int h0 = (blockIdx.y * kWaves + wave) * fit; h0 < steps; h0 += gridDim.y * kWaves * fit) {
    const int at = h0 + sub, t = p.tok == 1 ? 0 : at / heads, h = at - t * heads;
    const int64_t row = t0 + t;
    bool live = sub < fit && at < steps && row < a.tokens;
    const int side = h < a.n_heads ? 0 : h < a.n_heads + a.kv_heads ? 1 : 2;   // q, k, v
    const int hh = side == 0 ? h : h - a.n_heads - (side - 1) * a.kv_heads;
    if constexpr (APPEND) {   // rows that belong to no sequence stay as they are, in q_out too
      if (live) live = side == 0 ? row >= a.cu[0] && row < a.cu[a.n_seqs] : page_of[t] >= 0;
    }
    const T *src = (side == 0 ? (const T *)a.q + row * a.ldq : side == 1 ? (const T *)a.k + row * a.ldk : (const T *)a.v + row * a.ldv) + hh * dh + c0;
    float x[V];
    {
      u32x4 raw = {0, 0, 0, 0};
      if (live) raw = a.once ? __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(src)) : *reinterpret_cast<const u32x4 *>(src);
      widen<T>(raw, x);
    }
    if (norms) {
      const int kind = side == 2 ? PF_NORM_NONE : side == 0 ? a.norm[0].kind : a.norm[1].kind;
      const float eps = side == 0 ? a.norm[0].eps : a.norm[1].eps;
      const T *weight = (const T *)(side == 0 ? a.norm[0].weight : a.norm[1].weight), *bias = (const T *)(side == 0 ? a.norm[0].bias : a.norm[1].bias);
      const float inv = 1.0f / (float)dh;
      if (layer) {
        float t1 = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) t1 += x[i];
        const float mean = head.sum(t1) * inv;
        if (kind == PF_NORM_LAYER) {
#pragma unroll
          for (int i = 0; i < V; ++i) x[i] -= mean;
        }
      }
      float t2 = 0.f;
#pragma unroll
      for (int i = 0; i < V; ++i) t2 = fmaf(x[i], x[i], t2);
      t2 = head.sum(t2);
      if (kind != PF_NORM_NONE && live) {
        const float r = 1.0f / sqrtf(t2 * inv + eps);
        float w[V];
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] *= r;
        if (weight) {
          widen<T>(*reinterpret_cast<const u32x4 *>(weight + c0), w);
#pragma unroll
          for (int i = 0; i < V; ++i) x[i] *= w[i];
        }
        if (bias) {
          widen<T>(*reinterpret_cast<const u32x4 *>(bias + c0), w);
#pragma unroll
          for (int i = 0; i < V; ++i) x[i] += w[i];
        }
      }
    }
    if (rk.rot) {
      float y[V];
      if constexpr (HALF) {
        float *mine = other[wave] + sub * dh + c0;    // sub * dh + c0 + V <= 64 V
        if (sub < fit) {
#pragma unroll
          for (int i = 0; i < V; ++i) mine[i] = x[i];
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = sub < fit ? mine[i + (LAYOUT == TURN_HALVES ? to[0] : to[i])] : 0.f;
        __builtin_amdgcn_wave_barrier();
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = x[i ^ 1];
      }
      if (side != 2 && live) {
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (c0 + i < rk.rot) x[i] = fmaf(x[i], cosine[t][c0 + i], y[i] * sine[t][c0 + i]);
      }
    }
    // rounded to the rows' type, which is what the pages get too
    u32x4 raw;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 2) raw[i] = (unsigned)__builtin_bit_cast(unsigned short, (bf16_t)x[2 * i]) | (unsigned)__builtin_bit_cast(unsigned short, (bf16_t)x[2 * i + 1]) << 16;
      else raw[i] = __float_as_uint(x[i]);
    }
    if (!APPEND || side == 0) {
      T *dst = side == 0 ? (T *)a.q_out + row * a.ldqo + hh * dh + c0 : (T *)a.k_out + row * a.ldko + hh * dh + c0;
      if (live) *reinterpret_cast<u32x4 *>(dst) = raw;
    }
    if constexpr (APPEND) {
      widen<T>(raw, x);
      unsigned most = 0;
#pragma unroll
      for (int i = 0; i < V; ++i) most = max(most, __float_as_uint(x[i]) & 0x7fffffffu);
      constexpr int BL = PF_MX_BLOCK / V, BITS = Mx<FMT>::BITS;   // lanes of a block
      most = head.template group_max<BL>(most);
      if (side != 0 && live) {
        unsigned code[(V * BITS + 31) / 32];
        const unsigned byte = encode<FMT, V>(x, most, code);
        const int64_t in_page = ((int64_t)hh << a.pages.page_shift) + row_of[t];
        uint8_t *to_row = (side == 1 ? (uint8_t *)a.pages.k + page_of[t] * a.pages.k_stride : (uint8_t *)a.pages.v + page_of[t] * a.pages.v_stride) + in_page * a.mx.row_bytes;
        uint8_t *to_exp = (side == 1 ? a.mx.k_scale + page_of[t] * a.mx.k_scale_stride : a.mx.v_scale + page_of[t] * a.mx.v_scale_stride) + in_page * a.mx.blocks;
        uint8_t *dst = to_row + u * (V * BITS / 8);
        if constexpr (V * BITS == 64) *reinterpret_cast<u32x2 *>(dst) = u32x2{code[0], code[1]};
        else if constexpr (V * BITS == 32) *reinterpret_cast<unsigned *>(dst) = code[0];
        else *reinterpret_cast<unsigned short *>(dst) = (unsigned short)code[0];
        if (u % BL == 0) to_exp[u / BL] = (uint8_t)byte;
        if (u == n - 1)   // zeros up to whole 16 bytes: words, as head_dim is a multiple of 8
          for (int b = dh * BITS / 8; b < a.mx.row_bytes; b += 4) *reinterpret_cast<unsigned *>(to_row + b) = 0;
      }
    }
  }
}

// Slots of pages to rows: units of 16 bytes of a row, `tok` tokens to a workgroup.
struct ReadK {
  MxRead r;
  int tok, t0;
};
template <typename T, int FMT>
__global__ __launch_bounds__(256) void mx_read_kernel(ReadK p) {
  constexpr int V = 16 / (int)sizeof(T), BITS = Mx<FMT>::BITS;
  const MxRead &a = p.r;
  __shared__ int64_t page_of[16];       // -1: zeros; -2: the row belongs to no sequence
  __shared__ int row_of[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int t0 = p.t0 + blockIdx.x * p.tok, dh = a.head_dim;
  for (int t = wave; t < p.tok; t += 4) {
    int64_t page = -2;
    int in_page = 0;
    const int row = t0 + t;
    if (row < a.tokens) {
      const int s = wave_search(a.n_seqs, lane, row, [&](int i) { return a.cu[i]; });
      if (s >= 0 && s < a.n_seqs) {
        page = -1;
        const int64_t slot = (int64_t)a.first[s] + ((int64_t)row - a.cu[s]);
        if (slot >= 0 && slot < ((int64_t)a.pages.max_pages << a.pages.page_shift)) {
          const int pg = a.pages.table[(int64_t)s * a.pages.max_pages + (slot >> a.pages.page_shift)];
          if (pg >= 0 && pg < a.pages.n_pages) {
            page = pg;
            in_page = (int)(slot & ((1 << a.pages.page_shift) - 1));
          }
        }
      }
    }
    if (lane == 0) {
      page_of[t] = page;
      row_of[t] = in_page;
    }
  }
  __syncthreads();
  const int n = dh / V, per_side = a.kv_heads * n, per_token = ((a.k_out != nullptr) + (a.v_out != nullptr)) * per_side;
  for (int e = blockIdx.y * 256 + tid; e < p.tok * per_token; e += 256 * gridDim.y) {
    const int t = p.tok == 1 ? 0 : e / per_token, i = e - t * per_token;
    const int64_t page = page_of[t];
    if (page < -1) continue;
    const bool is_v = !a.k_out || i >= per_side;
    const int j = is_v && a.k_out ? i - per_side : i, h = j / n, u = j - h * n;
    T *dst = (is_v ? (T *)a.v_out + (t0 + t) * a.ldv : (T *)a.k_out + (t0 + t) * a.ldk) + (int64_t)h * dh + u * V;
    u32x4 raw = {0, 0, 0, 0};
    if (page >= 0) {
      const int64_t in_page = ((int64_t)h << a.pages.page_shift) + row_of[t];
      const uint8_t *row = (is_v ? (const uint8_t *)a.pages.v + page * a.pages.v_stride : (const uint8_t *)a.pages.k + page * a.pages.k_stride) + in_page * a.mx.row_bytes;
      const uint8_t *exp = (is_v ? a.mx.v_scale + page * a.mx.v_scale_stride : a.mx.k_scale + page * a.mx.k_scale_stride) + in_page * a.mx.blocks;
      const float power = mx_power(exp[u * V / PF_MX_BLOCK]);
      const uint8_t *src = row + u * (V * BITS / 8);
      unsigned w0, w1 = 0;
      if constexpr (V * BITS == 64) {
        const u32x2 x = *reinterpret_cast<const u32x2 *>(src);
        w0 = x[0], w1 = x[1];
      } else if constexpr (V * BITS == 32) {
        w0 = *reinterpret_cast<const unsigned *>(src);
      } else {
        w0 = *reinterpret_cast<const unsigned short *>(src);
      }
      if constexpr (sizeof(T) == 4) {
        const float2 lo = mx_decode_f32<FMT, 0>(w0, power), hi = mx_decode_f32<FMT, 1>(w0, power);
        raw = u32x4{__float_as_uint(lo.x), __float_as_uint(lo.y), __float_as_uint(hi.x), __float_as_uint(hi.y)};
      } else if constexpr (FMT == PF_MX_E4M3) {
        raw = u32x4{mx_decode_bf16<FMT, 0>(w0, power), mx_decode_bf16<FMT, 1>(w0, power), mx_decode_bf16<FMT, 0>(w1, power), mx_decode_bf16<FMT, 1>(w1, power)};
      } else {
        raw = u32x4{mx_decode_bf16<FMT, 0>(w0, power), mx_decode_bf16<FMT, 1>(w0, power), mx_decode_bf16<FMT, 2>(w0, power), mx_decode_bf16<FMT, 3>(w0, power)};
      }
    }
    *reinterpret_cast<u32x4 *>(dst) = raw;
  }
}

// Workgroups along y for launches of few tokens: a token's `parts` turns of a workgroup are split over them while they are few.
int split(int tokens, int parts) {
  int y = std::max(parts, 1);
  while (y > 1 && (int64_t)tokens * y > 4096) y = (y + 1) / 2;
  return y;
}

template <typename T, int FMT, int LAYOUT>
hipError_t launch_heads(const TurnK &rk, HeadsK p, hipStream_t s) {
  const int n = p.r.head_dim * (int)sizeof(T) / 16, per_turn = 64 / n * kWaves;
  const int heads = p.r.n_heads + (FMT >= 0 ? 2 : 1) * p.r.kv_heads, turns = (heads + per_turn - 1) / per_turn;
  p.tok = p.r.tokens >= 4096 && turns <= 1 ? 4 : p.r.tokens >= 4096 && turns <= 2 ? 2 : 1;
  const int y = p.tok == 1 ? split(p.r.tokens, turns) : 1;
  hipError_t e = hipSuccess;
  for (p.t0 = 0; p.t0 < p.r.tokens && e == hipSuccess; p.t0 += kLaunchRows) {
    const int rows = std::min(p.r.tokens - p.t0, kLaunchRows);
    head_rows_kernel<T, FMT, LAYOUT><<<dim3((rows + p.tok - 1) / p.tok, y), 64 * kWaves, 0, s>>>(rk, p);
    e = hipGetLastError();
  }
  return e;
}

template <typename T, int FMT>
hipError_t launch_layout(const TurnK &rk, const HeadsK &p, bool half, int align, hipStream_t s) {
  if (!half) return launch_heads<T, FMT, TURN_PAIRS>(rk, p, s);
  return align % (16 / (int)sizeof(T)) == 0 ? launch_heads<T, FMT, TURN_HALVES>(rk, p, s) : launch_heads<T, FMT, TURN_HALVES_ANY>(rk, p, s);
}
template <typename T>
hipError_t launch_format(const TurnK &rk, const HeadsK &p, bool half, int align, hipStream_t s) {
  if (!p.r.n_seqs) return launch_layout<T, -1>(rk, p, half, align, s);
  return p.r.mx.format == PF_MX_E4M3 ? launch_layout<T, PF_MX_E4M3>(rk, p, half, align, s) : launch_layout<T, PF_MX_E2M1>(rk, p, half, align, s);
}

template <typename T, int FMT>
hipError_t launch_read(ReadK p, hipStream_t s) {
  const int units = ((p.r.k_out != nullptr) + (p.r.v_out != nullptr)) * p.r.kv_heads * (p.r.head_dim * (int)sizeof(T) / 16);
  p.tok = p.r.tokens < 4096 || units >= 256 ? 1 : std::min(256 / units, 16);
  const int y = p.tok == 1 ? split(p.r.tokens, (units + 255) / 256) : 1;
  hipError_t e = hipSuccess;
  for (p.t0 = 0; p.t0 < p.r.tokens && e == hipSuccess; p.t0 += kLaunchRows) {
    const int rows = std::min(p.r.tokens - p.t0, kLaunchRows);
    mx_read_kernel<T, FMT><<<dim3((rows + p.tok - 1) / p.tok, y), 256, 0, s>>>(p);
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
