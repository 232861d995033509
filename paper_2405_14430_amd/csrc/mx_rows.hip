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

constexpr int kMaxPairs = PF_ROPE_MAX_PAIRS, kMaxDim = 128, kWaves = 4;
constexpr int V = 8;                                 // channels of a lane's unit
enum { TURN_PAIRS, TURN_HALVES, TURN_HALVES_ANY };   // neighbours; an axis' half apart, the halves whole fours of channels or not

struct TurnK {
  double turns[kMaxPairs];
  float magnitude;
  int n_axes, rot;                  // rot: channels that turn
  int axis_end[PF_ROPE_MAX_AXES];   // running end of the axes, in pairs
};

// The rows of q, k or v.
struct SideK {
  const void *src;
  void *dst;             // rows, or the first page of codes
  uint8_t *exp;          // the first page of exponents
  int64_t ld, ldo;
  const void *weight, *bias;
  int kind;
  float eps;
  int heads, steps;      // steps of a token
};
struct HeadsK {
  SideK side[3];
  int64_t code_stride[2], exp_stride[2];   // of the pages of k and v
  const int32_t *pos;
  Pages pages;
  const int32_t *cu, *first;
  int n_seqs, row_bytes, blocks;
  int tokens, head_dim;
  int t0;                // first token of the launch
};

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// A choice between values: `c ? a : b` of two arguments of a kernel is one of their addresses, from which lanes then load.
template <typename T>
__device__ __forceinline__ T pick(bool c, T a, T b) { return c ? a : b; }

// V channels of a row as they are in memory.
template <typename T>
struct Unit {
  static constexpr int N = V * (int)sizeof(T) / 16;
  u32x4 w[N];
  __device__ __forceinline__ void load(const T *p) {
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = reinterpret_cast<const u32x4 *>(p)[i];
  }
  __device__ __forceinline__ void store(T *p) const {
#pragma unroll
    for (int i = 0; i < N; ++i) reinterpret_cast<u32x4 *>(p)[i] = w[i];
  }
  __device__ __forceinline__ float operator[](int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i / 4][i % 4]);
    else return __uint_as_float(i & 1 ? w[0][i / 2] & 0xffff0000u : w[0][i / 2] << 16);
  }
  // The bits of the largest magnitude, as a float's; those of infinities and NaN are the largest.
  __device__ __forceinline__ unsigned largest() const {
    if constexpr (sizeof(T) == 2) {
      const auto mag = [&](int i) __attribute__((always_inline)) { return __builtin_bit_cast(u16x2, w[0][i] & 0x7fff7fffu); };
      const u16x2 m = __builtin_elementwise_max(__builtin_elementwise_max(mag(0), mag(1)), __builtin_elementwise_max(mag(2), mag(3)));
      return (unsigned)max(m[0], m[1]) << 16;
    } else {
      unsigned m = 0;
#pragma unroll
      for (int i = 0; i < V; ++i) m = max(m, w[i / 4][i % 4] & 0x7fffffffu);
      return m;
    }
  }
  // No magnitude past the float with bits `top` (a bf16 number).
  __device__ __forceinline__ void bound(unsigned top) {
    float x[V];
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = __builtin_amdgcn_fmed3f((*this)[i], -__uint_as_float(top), __uint_as_float(top));
    round(x);
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
  // The largest of the block of four lanes.  The last one of a head may be shorter: in place of a lane that is not there the head's last one is asked,
  // which lies in the same block (with itself in its place the second of three lanes would not hear of the third).
  __device__ __forceinline__ unsigned block_max(unsigned v) const {
    static_assert(PF_MX_BLOCK == 4 * V, "a block is four lanes");
    if constexpr (N != 0) {
      v = max(v, across<kSwap1>(v));
      return max(v, across<kSwap2>(v));
    }
#pragma unroll
    for (int o = 1; o < 4; o *= 2) v = max(v, (unsigned)__shfl((int)v, lane - u + min(u ^ o, n - 1), kWave));
    return v;
  }
};

// 1 / sqrt(x): the hardware's, within a unit, with a step of Newton's behind it.  Tiny sums are scaled, it takes no subnormal ones.
// (For bf16 rows, too: it moves a whole head, and each value next to a border of two codes that it takes across shows as a step of 2^-4.)
__device__ __forceinline__ float inverse_root(float x) {
  const bool tiny = x < 0x1p-100f;
  const float y = tiny ? x * 0x1p100f : x;
  float r = __builtin_amdgcn_rsqf(y);
  const float better = fmaf(0.5f * r, fmaf(-y * r, r, 1.0f), r);
  r = r == 0.f || y == 0.f ? r : better;
  return tiny ? r * 0x1p50f : r;
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

// Where packed row `row` of a call (one that all lanes agree on) goes in the pages: page (-1: none, -2: the row belongs to no sequence) and row
// of the page.  All loads are the scalar unit's: the vector unit's come back in order, so that one behind the rows' would wait for them.
__device__ __forceinline__ void find_slot(const Pages &pages, const int32_t *cu, const int32_t *first, int n_seqs, int row, int64_t &page, int &in_page) {
  page = -2;
  in_page = 0;
  int s = -1;                                 // the largest in [0, n_seqs] with cu[s] <= row
  for (int past = n_seqs + 1; past - s > 1;) {
    const int mid = (s + past) >> 1;
    if (cu[mid] <= row) s = mid;
    else past = mid;
  }
  if (s < 0 || s >= n_seqs) return;
  page = -1;
  const int64_t slot = (int64_t)first[s] + ((int64_t)row - cu[s]);
  if (slot < 0 || slot >= ((int64_t)pages.max_pages << pages.page_shift)) return;
  const int pg = pages.table[(int64_t)s * pages.max_pages + (slot >> pages.page_shift)];
  if (pg < 0 || pg >= pages.n_pages) return;
  page = pg;
  in_page = (int)(slot & ((1 << pages.page_shift) - 1));
}

// FMT < 0: q and k rows to rows; else k and v into pages.  LAYOUT: of the pairs.  N: lanes of a head (0: any number).
//
// A wave takes a token, or a share of its heads (gridDim.y shares): its 64 lanes work out the cosines and sines of up to 64 pairs and find the
// token's slot, then it goes over the heads, side after side (q, k, v), `fit` of them at a step.  A lane has the same channels of every head it
// meets, so their cosines, sines and weights stay in registers.  The rows of kDepth steps are loaded together, the first ones before
// all else; what hides a wave's waiting is the other waves, which it has nothing to do with.  (A workgroup over several tokens, their
// tables in LDS and their slots found together, took 57 us a call where this takes 49, 100 where 93, and 68 where 59.)
//   16896 tokens of 32 heads of 128, bf16, to rows: 277 MB in 45 us, 6.1 TB/s with the Infinity Cache's help.
//   16384 tokens of 72 heads of 64 into e4m3: 254 MB in 60 - 64 us, 4.1 TB/s; memory.
//   7178 tokens of 48 heads of 72, fp32, layer norm, halves, into e2m1: 144 MB in 46 us, 3.1 TB/s: waits for memory with 14 waves to a CU, whose
//   109 registers leave room for no more (bounded to 96 they spill: 63 us; two steps' loads at a time 47).
//   32 tokens of 40 heads of 128: 3.2 us in a graph, launch and two latencies.
template <typename T> constexpr int kDepth = sizeof(T) == 2 ? 4 : 3;
template <typename T, int FMT, int LAYOUT, int N>
__global__ __launch_bounds__(64 * kWaves) void head_rows_kernel(TurnK rk, HeadsK p) {
#pragma clang fp contract(off)   // the same rows from all instances: pages get what pf_op_qk_norm_rope gives
  constexpr bool APPEND = FMT >= 0, HALF = LAYOUT != TURN_PAIRS;
  constexpr int DEPTH = kDepth<T>;
  __shared__ __attribute__((aligned(16))) float table[kWaves][2][kMaxDim];                      // cosines and sines by channel
  __shared__ __attribute__((aligned(16))) float other[HALF ? kWaves : 1][HALF ? 64 * V : 1];   // the wave's units, for the pairs' other channels
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int token = p.t0 + blockIdx.x * kWaves + wave;
  if (token >= p.tokens) return;

  const int dh = N ? N * V : p.head_dim, n = N ? N : dh / V, fit = 64 / n;   // channels and lanes of a head, heads of a step
  const int sub = lane / n, u = lane - sub * n, c0 = u * V;                  // the lane's head of these, unit and first channel
  const HeadLanes<N> head{lane, u, n};
  const int q_steps = p.side[0].steps, k_steps = p.side[1].steps, steps = q_steps + (APPEND ? 2 : 1) * k_steps;
  const int stride = gridDim.y;
  const T *const q = (const T *)p.side[0].src + token * p.side[0].ld, *const k = (const T *)p.side[1].src + token * p.side[1].ld;
  const T *const v = (const T *)p.side[2].src + token * p.side[2].ld;
  // of step i: side, first head, lanes that have a head
  struct Where {
    int side, h0, lanes;
  };
  const auto where = [&](int i) __attribute__((always_inline)) {
    Where x;
    x.side = i < q_steps ? 0 : !APPEND || i < q_steps + k_steps ? 1 : 2;
    x.h0 = (i - (x.side == 0 ? 0 : x.side == 1 ? q_steps : q_steps + k_steps)) * fit;
    x.lanes = min(fit, pick(x.side == 0, p.side[0].heads, p.side[1].heads) - x.h0) * n;
    return x;
  };
  int64_t page = 0;
  int in_page = 0;
  if constexpr (APPEND) {
    find_slot(p.pages, p.cu, p.first, p.n_seqs, token, page, in_page);
    if (page == -2) return;           // rows that belong to no sequence stay as they are, in q_out too
  }
  Unit<T> raw[DEPTH];
#pragma unroll
  for (int j = 0; j < DEPTH; ++j)
#pragma unroll
    for (int i = 0; i < Unit<T>::N; ++i) {
      raw[j].w[i] = u32x4{0, 0, 0, 0};                      // lanes without a head
      asm volatile("" : "+v"(raw[j].w[i]));                 // four registers that stay together
    }
  const auto load = [&](int i) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < DEPTH; ++j, i += stride) {
      if (i >= steps) break;
      const Where at = where(i);
      if (lane < at.lanes) raw[j].load(pick(at.side == 0, q, pick(at.side == 1, k, v)) + at.h0 * dh + lane * V);
    }
  };
  load(blockIdx.y);
  Unit<T> weight[2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (p.side[i].weight) weight[i].load((const T *)p.side[i].weight + c0);

  // the token's cosines and sines, a lane to a pair, and from there to the lanes of its channels
  float cs[V], sn[V];
  if (rk.rot) {
    if (2 * lane < rk.rot) {
      const int end0 = rk.axis_end[0], end1 = rk.axis_end[1];
      const int axis = (lane >= end0) + (rk.n_axes > 1 && lane >= end1);
      const double turns = (double)p.pos[(int64_t)token * rk.n_axes + axis] * rk.turns[lane];
      const double part = turns - rint(turns);
      float sin0, cos0;
      sincospif(2.0f * (float)part, &sin0, &cos0);
      const float rest = (float)((part - (float)part) * 6.283185307179586);   // what 24 bits of the fraction leave out, in radians
      const float s = fmaf(cos0, rest, sin0), c = fmaf(-sin0, rest, cos0);
      const int begin = pick(axis == 0, 0, pick(axis == 1, end0, end1)), w = pick(axis == 0, end0, pick(axis == 1, end1, rk.axis_end[2])) - begin;
      const int one = HALF ? 2 * begin + (lane - begin) : 2 * lane, two = HALF ? one + w : one + 1;
      table[wave][0][one] = table[wave][0][two] = c * rk.magnitude;
      table[wave][1][one] = -s * rk.magnitude;
      table[wave][1][two] = s * rk.magnitude;
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int c = 0; c < V; c += 4) {
      const float4 x = *reinterpret_cast<const float4 *>(&table[wave][0][c0 + c]), y = *reinterpret_cast<const float4 *>(&table[wave][1][c0 + c]);
      cs[c] = x.x, cs[c + 1] = x.y, cs[c + 2] = x.z, cs[c + 3] = x.w;
      sn[c] = y.x, sn[c + 1] = y.y, sn[c + 2] = y.z, sn[c + 3] = y.w;
    }
  }
  const float inv = 1.0f / (float)dh;
  // where the pairs' other channels are, from the lane's own, for GROUP neighbouring channels each
  constexpr int GROUP = LAYOUT == TURN_HALVES ? 4 : 1;
  int to[V / GROUP];
  if constexpr (HALF) {
#pragma unroll
    for (int i = 0; i < V / GROUP; ++i) {
      const int c = c0 + i * GROUP, e0 = 2 * rk.axis_end[0], e1 = rk.n_axes > 1 ? 2 * rk.axis_end[1] : rk.rot;
      const int begin = c < e0 ? 0 : c < e1 ? e0 : e1, end = c < e0 ? e0 : c < e1 ? e1 : rk.rot, w = (end - begin) >> 1;
      to[i] = c >= rk.rot ? 0 : c < begin + w ? w : -w;
    }
  }
  // the lane's bytes of codes and its block's exponent from a step's first head on
  constexpr int BYTES = APPEND ? V * Mx<APPEND ? FMT : 0>::BITS / 8 : 0;
  const int code_off = APPEND ? (sub << p.pages.page_shift) * p.row_bytes + u * BYTES : 0;
  const int exp_off = APPEND ? (sub << p.pages.page_shift) * p.blocks + u / 4 : 0;

  for (int i0 = blockIdx.y;;) {
    // all rows are waited for here: in front of a later step the wait would be one for the stores of the step before, too
#pragma unroll
    for (int j = 0; j < DEPTH; ++j)
#pragma unroll
      for (int c = 0; c < Unit<T>::N; ++c) asm volatile("" : "+v"(raw[j].w[c]));
#pragma unroll
    for (int j = 0; j < DEPTH; ++j) {
      const int i = i0 + j * stride;
      if (i >= steps) break;
      const Where at = where(i);
      if (APPEND && at.side != 0 && page < 0) break;
      Unit<T> &unit = raw[j];
      if (at.side != 2) {
        float x[V];
#pragma unroll
        for (int c = 0; c < V; ++c) x[c] = unit[c];
        const bool is_q = at.side == 0;
        const int kind = pick(is_q, p.side[0].kind, p.side[1].kind);
        const float eps = pick(is_q, p.side[0].eps, p.side[1].eps);
        const T *const w = (const T *)pick(is_q, p.side[0].weight, p.side[1].weight), *const b = (const T *)pick(is_q, p.side[0].bias, p.side[1].bias);
        if (kind != PF_NORM_NONE) {
          if (kind == PF_NORM_LAYER) {
            float sum = 0.f;
#pragma unroll
            for (int c = 0; c < V; ++c) sum += x[c];
            const float mean = head.sum(sum) * inv;
#pragma unroll
            for (int c = 0; c < V; ++c) x[c] -= mean;
          }
          float sum = 0.f;
#pragma unroll
          for (int c = 0; c < V; ++c) sum = fmaf(x[c], x[c], sum);
          const float r = inverse_root(fmaf(head.sum(sum), inv, eps));
          if (w) {                                    // in front of r: a product of two bf16 numbers is exact
            Unit<T> g;
#pragma unroll
            for (int c = 0; c < Unit<T>::N; ++c) g.w[c] = pick(is_q, weight[0].w[c], weight[1].w[c]);
#pragma unroll
            for (int c = 0; c < V; ++c) x[c] *= g[c];
          }
#pragma unroll
          for (int c = 0; c < V; ++c) x[c] *= r;
          if (b) {
            Unit<T> bias;
            bias.load(b + c0);
#pragma unroll
            for (int c = 0; c < V; ++c) x[c] += bias[c];
          }
        }
        if (rk.rot) {
          float y[V], z[V];
          if constexpr (HALF) {
            float *mine = other[wave] + lane * V;     // a head's units are dh floats
#pragma unroll
            for (int c = 0; c < V; c += 4) *reinterpret_cast<float4 *>(mine + c) = make_float4(x[c], x[c + 1], x[c + 2], x[c + 3]);
            __builtin_amdgcn_wave_barrier();
            if (lane < fit * n) {                     // behind the last head there is no other channel
              if constexpr (LAYOUT == TURN_HALVES) {
#pragma unroll
                for (int c = 0; c < V; c += 4) {
                  const float4 o = *reinterpret_cast<const float4 *>(mine + c + to[c / 4]);
                  y[c] = o.x, y[c + 1] = o.y, y[c + 2] = o.z, y[c + 3] = o.w;
                }
              } else {
#pragma unroll
                for (int c = 0; c < V; ++c) y[c] = mine[c + to[c]];
              }
            }
            __builtin_amdgcn_wave_barrier();
          } else {
#pragma unroll
            for (int c = 0; c < V; ++c) y[c] = x[c ^ 1];
          }
#pragma unroll
          for (int c = 0; c < V; ++c) z[c] = fmaf(x[c], cs[c], y[c] * sn[c]);
          if (rk.rot == dh) {
#pragma unroll
            for (int c = 0; c < V; ++c) x[c] = z[c];
          } else {
#pragma unroll
            for (int c = 0; c < V; ++c) x[c] = c0 + c < rk.rot ? z[c] : x[c];
          }
        }
        unit.round(x);   // to the rows' type, which is what the pages get too
      }
      if (!APPEND || at.side == 0) {
        const bool is_q = at.side == 0;
        T *dst = (T *)pick(is_q, p.side[0].dst, p.side[1].dst) + token * pick(is_q, p.side[0].ldo, p.side[1].ldo) + at.h0 * dh;
        if (lane < at.lanes) unit.store(dst + lane * V);
      } else if constexpr (APPEND) {
        unsigned code[2];
        const unsigned byte = mx_encode<FMT>(unit, head.block_max(unit.largest()), code);
        if (lane < at.lanes) {
          const bool is_v = at.side == 2;
          const int64_t row = ((int64_t)at.h0 << p.pages.page_shift) + in_page;
          uint8_t *to_row = (uint8_t *)pick(is_v, p.side[2].dst, p.side[1].dst) + (page * pick(is_v, p.code_stride[1], p.code_stride[0]) + row * p.row_bytes) + code_off;
          uint8_t *to_exp = pick(is_v, p.side[2].exp, p.side[1].exp) + (page * pick(is_v, p.exp_stride[1], p.exp_stride[0]) + row * p.blocks) + exp_off;
          if constexpr (BYTES == 8) *reinterpret_cast<u32x2 *>(to_row) = u32x2{code[0], code[1]};
          else *reinterpret_cast<unsigned *>(to_row) = code[0];
          if (u % 4 == 0) *to_exp = (uint8_t)byte;
          if (N == 0 && u == n - 1)   // zeros up to whole 16 bytes: words, as head_dim is a multiple of 8
            for (int b = n * BYTES; b < p.row_bytes; b += 4) *reinterpret_cast<unsigned *>(to_row + (b - u * BYTES)) = 0;
        }
      }
    }
    i0 += DEPTH * stride;
    if (i0 >= steps) return;
    load(i0);
  }
}

// Slots of pages to rows: a workgroup takes tok tokens, a wave `fit` heads at a step and READ_DEPTH steps' loads at a time.  Bound by memory:
// 24 caches of up to 8192 tokens, 8 heads of 128, e4m3 to bf16, 221 MB in 40 us, 5.5 TB/s.
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
    if (t0 + t < a.tokens) find_slot(a.pages, a.cu, a.first, a.n_seqs, t0 + t, page, in_page);
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

// Workgroups along y for launches of few tokens: a token's `parts` turns of a workgroup are split over them while they are few.  Up to 4096 shares:
// 1024 tokens of 40 heads of 128 are normed and turned in 6.8 us (up to 2048: 7.5, 16384: 7.7, tokens left whole: 9.5), 8 tokens in 3.2 (whole: 7.9), 4096 in
// 17.7 either way.
int split(int tokens, int parts) {
  int y = std::max(parts, 1);
  while (y > 1 && (int64_t)tokens * y > 4096) y = (y + 1) / 2;
  return y;
}

template <typename T, int FMT, int LAYOUT, int N>
hipError_t launch_heads(const TurnK &rk, HeadsK p, hipStream_t s) {
  int steps = 0;         // of a token
  for (const SideK &side : p.side) steps += side.steps;
  const int y = split(p.tokens, steps);
  hipError_t e = hipSuccess;
  for (p.t0 = 0; p.t0 < p.tokens && e == hipSuccess; p.t0 += kLaunchRows) {
    const int rows = std::min(p.tokens - p.t0, kLaunchRows);
    head_rows_kernel<T, FMT, LAYOUT, N><<<dim3((rows + kWaves - 1) / kWaves, y), 64 * kWaves, 0, s>>>(rk, p);
    e = hipGetLastError();
  }
  return e;
}

template <typename T, int FMT, int LAYOUT>
hipError_t launch_lanes(const TurnK &rk, const HeadsK &p, hipStream_t s) {
  if (p.head_dim == 128) return launch_heads<T, FMT, LAYOUT, 16>(rk, p, s);
  if (p.head_dim == 64) return launch_heads<T, FMT, LAYOUT, 8>(rk, p, s);
  return launch_heads<T, FMT, LAYOUT, 0>(rk, p, s);
}
template <typename T, int FMT>
hipError_t launch_layout(const TurnK &rk, const HeadsK &p, bool half, int align, hipStream_t s) {
  if (half && align % 4) return launch_heads<T, FMT, TURN_HALVES_ANY, 0>(rk, p, s);
  return half ? launch_lanes<T, FMT, TURN_HALVES>(rk, p, s) : launch_lanes<T, FMT, TURN_PAIRS>(rk, p, s);
}
template <typename T>
hipError_t launch_format(const TurnK &rk, const HeadsK &p, int format, bool half, int align, hipStream_t s) {
  if (format < 0) return launch_layout<T, -1>(rk, p, half, align, s);
  return format == PF_MX_E4M3 ? launch_layout<T, PF_MX_E4M3>(rk, p, half, align, s) : launch_layout<T, PF_MX_E2M1>(rk, p, half, align, s);
}

template <typename T, int FMT>
hipError_t launch_read(ReadK p, hipStream_t s) {
  const int per_turn = 64 / (p.r.head_dim / V) * kWaves, heads = ((p.r.k_out != nullptr) + (p.r.v_out != nullptr)) * p.r.kv_heads;
  // one token to a workgroup, its heads split, or several: 1024 tokens of 2 x 8 heads of 128 4.5 and 4.7 us, 2048 6.3 and 5.9, 4096 9.6 and 8.0
  p.tok = p.r.tokens < 2048 ? 1 : std::min(std::max(READ_DEPTH * per_turn / heads, 1), kMaxReadTok);
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
  const bool append = args.n_seqs > 0;
  const int fit = 64 / (args.head_dim / V);
  const auto side = [&](const void *src, int64_t ld, void *dst, int64_t ldo, uint8_t *exp, const NormSide &n, int heads) {
    return SideK{src, dst, exp, ld, ldo, n.weight, n.bias, n.kind, n.eps, heads, (heads + fit - 1) / fit};
  };
  HeadsK p{};
  p.side[0] = side(args.q, args.ldq, args.q_out, args.ldqo, nullptr, args.norm[0], args.n_heads);
  p.side[1] = side(args.k, args.ldk, append ? args.pages.k : args.k_out, args.ldko, args.mx.k_scale, args.norm[1], args.kv_heads);
  if (append) p.side[2] = side(args.v, args.ldv, args.pages.v, 0, args.mx.v_scale, NormSide{}, args.kv_heads);
  p.code_stride[0] = args.pages.k_stride, p.code_stride[1] = args.pages.v_stride;
  p.exp_stride[0] = args.mx.k_scale_stride, p.exp_stride[1] = args.mx.v_scale_stride;
  p.pos = args.pos, p.pages = args.pages, p.cu = args.cu, p.first = args.first, p.n_seqs = args.n_seqs;
  p.row_bytes = args.mx.row_bytes, p.blocks = args.mx.blocks, p.tokens = args.tokens, p.head_dim = args.head_dim;
  const int format = append ? args.mx.format : -1;
  return args.dt == DT_BF16 ? launch_format<bf16_t>(rk, p, format, half, align, s) : launch_format<float>(rk, p, format, half, align, s);
}

hipError_t launch_mx_read(const MxRead &r, hipStream_t s) {
  if (r.tokens <= 0) return hipSuccess;
  const ReadK p{r, 1, 0};
  if (r.dt == DT_BF16) return r.mx.format == PF_MX_E4M3 ? launch_read<bf16_t, PF_MX_E4M3>(p, s) : launch_read<bf16_t, PF_MX_E2M1>(p, s);
  return r.mx.format == PF_MX_E4M3 ? launch_read<float, PF_MX_E4M3>(p, s) : launch_read<float, PF_MX_E2M1>(p, s);
}

}  // namespace pf
