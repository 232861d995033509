// The rows between two branches of a block in one pass: norm of the branch's output, gate, residual, norm and modulation for the
// next branch,
//   x' = x_scale x + g(gate) (post(y) w + b),    h = (pre(x') w + b) (1 + scale) + shift,
// with RMS or Layer norms over a row and gate / scale / shift vectors per sequence.
//
// Bound by memory: y and x are read once, x' and h written once, a row lives in registers between its (up to four) sums.
// 16384 fp32 rows of 1152 with both norms, gate and modulation, from memory: 58 us, 302 MB at 5.2 TB/s, a large device copy's rate
// or better; 32 rows of 1536: 4.5 us between two calls of a graph, launch, one wait for memory and three sums behind each other.
// A row belongs to one wave, or to 2, 4 or 8 that add their sums up through LDS (the rule and what it measured: at the launch).
// The variance is the mean of (x - mean)^2 over the registers, a second sum and no difference of squares.  Sums in 32 bits.
#include <algorithm>
#include <type_traits>

#include "requests.h"

namespace pf {
namespace {

constexpr int kLayer = PF_NORM_LAYER;

template <typename T, bool ONCE = false> __device__ __forceinline__ void load4(const T *p, float *o) {
  using V = std::conditional_t<sizeof(T) == 2, bf16x4, f32x4>;
  const V v = ONCE ? __builtin_nontemporal_load(reinterpret_cast<const V *>(p)) : *reinterpret_cast<const V *>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = (float)v[i];
}
template <typename T> __device__ __forceinline__ void store4(T *p, const float *o) {
  if constexpr (sizeof(T) == 2) {
    bf16x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (bf16_t)o[i];
    *reinterpret_cast<bf16x4 *>(p) = v;
  } else {
    *reinterpret_cast<float4 *>(p) = make_float4(o[0], o[1], o[2], o[3]);
  }
}

// Sum over the W waves of a row; `part` is the row's own W floats of LDS, a different one for every sum of a row.
template <int W>
__device__ __forceinline__ float row_sum(float v, int wave, int lane, float *part) {
  v = wave_sum(v);
  if constexpr (W > 1) {
    if (lane == 0) part[wave] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) v += part[i];
  }
  return v;
}

// NV groups of four channels per lane; W waves per row, as many rows as fit a workgroup of max(W, 4) waves.
template <typename T, int NV, int W>
__global__ __launch_bounds__(64 * (W < 4 ? 4 : W)) void norm_residual_kernel(NormResidual a) {
  constexpr int WAVES = W < 4 ? 4 : W, RPB = WAVES / W;
  __shared__ float part[4][RPB][W];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int slot = wave / W, wr = wave % W;
  // W > 1: every wave of the workgroup reaches every barrier, so a row past the end is worked on as a copy and not stored
  const int64_t row_at = a.row0 + (int64_t)blockIdx.x * RPB + slot;
  bool live = row_at < a.rows;
  const int64_t row = live ? row_at : a.rows - 1;
  int seg = 0;
  if (a.cu) {
    seg = wave_search(a.n_seqs, lane, row, [&](int i) { return a.cu[i]; });
    if (seg < 0 || seg >= a.n_seqs) {   // rows of no sequence stay as they are
      live = false;
      seg = 0;
    }
  }
  const int d = a.d, c0 = (wr * 64 + lane) * 4;
  constexpr int STEP = W * 64 * 4;
  const float inv_d = 1.0f / (float)d;

  // The vectors of the two norms, the gate and the modulation do not depend on the row's sums: with up to two groups per lane they
  // are loaded in front of the first one, so that a launch of few rows waits for memory once and not once per sum (32
  // rows of 4096, bf16: 5.1 -> 4.8 us).  With three or four groups their registers leave too few waves (16384 rows of 1152: 44 -> 56).
  constexpr bool EARLY = NV <= 2;
  struct Vectors {
    float wy[NV][4], by[NV][4], g[NV][4], wx[NV][4], bx[NV][4], sc[NV][4], sh[NV][4];
  } vec;
  const float *gp = a.gate ? a.gate + seg * a.gate_stride : nullptr;
  const float *scp = a.scale ? a.scale + seg * a.mod_stride : nullptr, *shp = a.shift ? a.shift + seg * a.mod_stride : nullptr;
  auto get_as = [&](auto once, auto *p, float (&o)[4], int c, float none) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = none;
    if (p && c < d) load4<std::remove_const_t<std::remove_pointer_t<decltype(p)>>, decltype(once)::value>(p + c, o);
  };
  auto get = [&](auto *p, float (&o)[4], int c, float none) __attribute__((always_inline)) { get_as(std::false_type{}, p, o, c, none); };
  const T *wyp = (const T *)a.post.weight, *byp = (const T *)a.post.bias, *wxp = (const T *)a.pre.weight, *bxp = (const T *)a.pre.bias;

  float x[NV][4], y[NV][4];
  const float *xp = a.x + row * a.ldx;
  const T *yp = a.y ? (const T *)a.y + row * a.ldy : nullptr;
  auto rows = [&](auto once) __attribute__((always_inline)) {
#pragma unroll
    for (int v = 0; v < NV; ++v) get_as(once, xp, x[v], c0 + v * STEP, 0.f);
#pragma unroll
    for (int v = 0; v < NV; ++v) get_as(once, yp, y[v], c0 + v * STEP, 0.f);
  };
  if (a.once) rows(std::true_type{});
  else rows(std::false_type{});
  if constexpr (EARLY) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = c0 + v * STEP;
      get(wyp, vec.wy[v], c, 1.f);
      get(byp, vec.by[v], c, 0.f);
      get(gp, vec.g[v], c, 1.f);
      get(wxp, vec.wx[v], c, 1.f);
      get(bxp, vec.bx[v], c, 0.f);
      get(scp, vec.sc[v], c, 0.f);
      get(shp, vec.sh[v], c, 0.f);
    }
  }
  if (a.y) {
    if (a.post.kind != PF_NORM_NONE) {
      float mean = 0.f;
      if (a.post.kind == kLayer) {
        float t = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v) t += (y[v][0] + y[v][1]) + (y[v][2] + y[v][3]);
        mean = row_sum<W>(t, wr, lane, part[0][slot]) * inv_d;
      }
      float t = 0.f;
#pragma unroll
      for (int v = 0; v < NV; ++v)
        if (c0 + v * STEP < d) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            y[v][i] -= mean;
            t = fmaf(y[v][i], y[v][i], t);
          }
        }
      const float r = 1.0f / sqrtf(row_sum<W>(t, wr, lane, part[1][slot]) * inv_d + a.post.eps);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        if constexpr (!EARLY) {
          get(wyp, vec.wy[v], c0 + v * STEP, 1.f);
          get(byp, vec.by[v], c0 + v * STEP, 0.f);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) y[v][i] = fmaf(y[v][i] * r, vec.wy[v][i], vec.by[v][i]);
      }
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if constexpr (!EARLY) get(gp, vec.g[v], c0 + v * STEP, 1.f);
      if (gp && a.gate_tanh) {
#pragma unroll
        for (int i = 0; i < 4; ++i) vec.g[v][i] = tanhf(vec.g[v][i]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) x[v][i] = fmaf(vec.g[v][i], y[v][i], a.x_scale * x[v][i]);
    }
  } else {
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < 4; ++i) x[v][i] *= a.x_scale;
  }
  if (a.x_out && live) {
    float *op = a.x_out + row * a.ldxo;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (c0 + v * STEP < d) store4(op + c0 + v * STEP, x[v]);
  }
  if (!a.h) return;

  float mean = 0.f, r = 1.f;
  if (a.pre.kind != PF_NORM_NONE) {
    if (a.pre.kind == kLayer) {
      float t = 0.f;
#pragma unroll
      for (int v = 0; v < NV; ++v)
        if (c0 + v * STEP < d) t += (x[v][0] + x[v][1]) + (x[v][2] + x[v][3]);
      mean = row_sum<W>(t, wr, lane, part[2][slot]) * inv_d;
    }
    float t = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (c0 + v * STEP < d) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[v][i] -= mean;
          t = fmaf(x[v][i], x[v][i], t);
        }
      }
    r = 1.0f / sqrtf(row_sum<W>(t, wr, lane, part[3][slot]) * inv_d + a.pre.eps);
  }
  if (!live) return;
  T *hp = (T *)a.h + row * a.ldh;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = c0 + v * STEP;
    if constexpr (!EARLY) {
      get(wxp, vec.wx[v], c, 1.f);
      get(bxp, vec.bx[v], c, 0.f);
      get(scp, vec.sc[v], c, 0.f);
      get(shp, vec.sh[v], c, 0.f);
    }
    if (c < d) {
      float o[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        o[i] = fmaf(x[v][i] * r, vec.wx[v][i], vec.bx[v][i]);
        o[i] = fmaf(o[i], vec.sc[v][i], o[i]) + vec.sh[v][i];
      }
      store4(hp + c, o);
    }
  }
}

template <typename T, int NV, int W>
hipError_t launch_nw(NormResidual a, hipStream_t s) {
  constexpr int WAVES = W < 4 ? 4 : W, RPB = WAVES / W;
  static_assert(kLaunchRows % RPB == 0, "a launch ends with whole workgroups");
  hipError_t e = hipSuccess;
  for (a.row0 = 0; a.row0 < a.rows && e == hipSuccess; a.row0 += kLaunchRows) {
    const int n = std::min(a.rows - a.row0, kLaunchRows);
    norm_residual_kernel<T, NV, W><<<dim3((n + RPB - 1) / RPB), 64 * WAVES, 0, s>>>(a);
    e = hipGetLastError();
  }
  return e;
}

template <typename T, int W>
hipError_t launch_w(const NormResidual &a, hipStream_t s) {
  const int nv = (a.d / 4 + 64 * W - 1) / (64 * W);
  if (nv <= 1) return launch_nw<T, 1, W>(a, s);
  if (nv <= 2) return launch_nw<T, 2, W>(a, s);
  if (nv <= 3) return launch_nw<T, 3, W>(a, s);
  return launch_nw<T, 4, W>(a, s);
}

}  // namespace

hipError_t launch_norm_residual(const NormResidual &args, hipStream_t s) {
  if (args.rows <= 0) return hipSuccess;
  NormResidual a = args;
  const int64_t el = (int64_t)dt_size(a.dt);
  a.once = (int64_t)a.rows * a.d * (4 + (a.y ? el : 0) + (a.x_out ? 4 : 0) + (a.h ? el : 0)) > kReadOnceBytes;
  // Waves per row: so many that a lane holds at most four groups of four channels of each row it works on (16384 rows, bf16, in
  // us: up to eight groups, up to four, up to two: 1536 channels 84, 60, 75; 4096: 227, 172, 202; 8192: 444, 337, 337; fp32: 1536: 74,
  // 68, 72), and twice or four times as many while the launch has fewer than 4096 waves and a wave still has two groups per
  // lane (32 rows of 1536, bf16: 4.5 us with four waves, 9.0 with one; 1024 rows of 4096: 13.2, up to 2048 waves 16.4, up to 8192
  // 14.3; 4000 rows of 1152: 13.4 with two, 18.8 with four).
  int w = 1;
  while (a.d > w * 1024) w *= 2;
  while (w < 8 && (int64_t)a.rows * w < 4096 && a.d > w * 512) w *= 2;
  if (a.dt == DT_BF16)
    return w == 1 ? launch_w<bf16_t, 1>(a, s) : w == 2 ? launch_w<bf16_t, 2>(a, s) : w == 4 ? launch_w<bf16_t, 4>(a, s) : launch_w<bf16_t, 8>(a, s);
  return w == 1 ? launch_w<float, 1>(a, s) : w == 2 ? launch_w<float, 2>(a, s) : w == 4 ? launch_w<float, 4>(a, s) : launch_w<float, 8>(a, s);
}

}  // namespace pf
