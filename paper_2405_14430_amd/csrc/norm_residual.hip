// The rows between two branches of a block in one pass: norm of the branch's output, gate, residual, norm and modulation for the
// next branch,
//   x' = x_scale x + g(gate) (post(y) w + b),    h = (pre(x') w + b) (1 + scale) + shift,
// with RMS or Layer norms over a row and gate / scale / shift vectors per sequence.
//
// Bound by memory: y and x are read once, x' and h written once, a row lives in registers between its (up to four) sums.
// A row belongs to one wave, or to 2, 4 or 8 that add their sums up through LDS: few rows need the waves, many rows do not.
// The variance is the mean of (x - mean)^2 over the registers, a second sum and no difference of squares.  Sums in 32 bits.
#include "requests.h"

namespace pf {
namespace {

constexpr int kLayer = PF_NORM_LAYER;

template <typename T> __device__ __forceinline__ void load4(const T *p, float *o) {
  if constexpr (sizeof(T) == 2) {
    const bf16x4 v = *reinterpret_cast<const bf16x4 *>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = (float)v[i];
  } else {
    const float4 v = *reinterpret_cast<const float4 *>(p);
    o[0] = v.x; o[1] = v.y; o[2] = v.z; o[3] = v.w;
  }
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

// NV groups of four channels per lane; W waves per row, 8 / W rows (at least one) per workgroup of max(W, 4) waves.
template <typename T, int NV, int W>
__global__ __launch_bounds__(64 * (W < 4 ? 4 : W)) void norm_residual_kernel(NormResidual a) {
  constexpr int WAVES = W < 4 ? 4 : W, RPB = WAVES / W;
  __shared__ float part[4][RPB][W];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int slot = wave / W, wr = wave % W;
  // W > 1: every wave of the workgroup reaches every barrier, so a row past the end is worked on as a copy and not stored
  const int64_t row_at = (int64_t)blockIdx.x * RPB + slot;
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

  float x[NV][4];
  const float *xp = a.x + row * a.ldx;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = c0 + v * STEP;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[v][i] = 0.f;
    if (c < d) load4(xp + c, x[v]);
  }
  if (a.y) {
    float y[NV][4];
    const T *yp = (const T *)a.y + row * a.ldy;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = c0 + v * STEP;
#pragma unroll
      for (int i = 0; i < 4; ++i) y[v][i] = 0.f;
      if (c < d) load4(yp + c, y[v]);
    }
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
        const int c = c0 + v * STEP;
        if (c < d) {
          float w[4] = {1.f, 1.f, 1.f, 1.f}, b[4] = {0.f, 0.f, 0.f, 0.f};
          if (a.post.weight) load4((const T *)a.post.weight + c, w);
          if (a.post.bias) load4((const T *)a.post.bias + c, b);
#pragma unroll
          for (int i = 0; i < 4; ++i) y[v][i] = fmaf(y[v][i] * r, w[i], b[i]);
        }
      }
    }
    const float *gp = a.gate ? a.gate + seg * a.gate_stride : nullptr;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = c0 + v * STEP;
      if (c < d) {
        float g[4] = {1.f, 1.f, 1.f, 1.f};
        if (gp) {
          load4(gp + c, g);
          if (a.gate_tanh) {
#pragma unroll
            for (int i = 0; i < 4; ++i) g[i] = tanhf(g[i]);
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) x[v][i] = fmaf(g[i], y[v][i], a.x_scale * x[v][i]);
      }
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
      for (int v = 0; v < NV; ++v) t += (x[v][0] + x[v][1]) + (x[v][2] + x[v][3]);
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
  const float *sc = a.scale ? a.scale + seg * a.mod_stride : nullptr, *sh = a.shift ? a.shift + seg * a.mod_stride : nullptr;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = c0 + v * STEP;
    if (c < d) {
      float w[4] = {1.f, 1.f, 1.f, 1.f}, b[4] = {0.f, 0.f, 0.f, 0.f}, o[4];
      if (a.pre.weight) load4((const T *)a.pre.weight + c, w);
      if (a.pre.bias) load4((const T *)a.pre.bias + c, b);
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = fmaf(x[v][i] * r, w[i], b[i]);
      if (sc) {
        load4(sc + c, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = fmaf(o[i], w[i], o[i]);
      }
      if (sh) {
        load4(sh + c, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] += b[i];
      }
      store4(hp + c, o);
    }
  }
}

template <typename T, int NV, int W>
hipError_t launch_nw(const NormResidual &a, hipStream_t s) {
  constexpr int WAVES = W < 4 ? 4 : W, RPB = WAVES / W;
  norm_residual_kernel<T, NV, W><<<dim3((a.rows + RPB - 1) / RPB), 64 * WAVES, 0, s>>>(a);
  return hipGetLastError();
}

template <typename T, int W>
hipError_t launch_w(const NormResidual &a, hipStream_t s) {
  const int nv = (a.d / 4 + 64 * W - 1) / (64 * W);
  if (nv <= 1) return launch_nw<T, 1, W>(a, s);
  if (nv <= 2) return launch_nw<T, 2, W>(a, s);
  if (nv <= 3) return launch_nw<T, 3, W>(a, s);
  if (nv <= 5) return launch_nw<T, 5, W>(a, s);
  return launch_nw<T, 8, W>(a, s);
}

}  // namespace

hipError_t launch_norm_residual(const NormResidual &a, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  // Waves per row: enough that a lane holds at most eight groups of four channels, and twice or four times as many while
  // the launch has fewer than 4096 waves and a wave still has two groups per lane.
  int w = 1;
  while (a.d > w * 2048) w *= 2;
  while (w < 8 && (int64_t)a.rows * w < 4096 && a.d > w * 512) w *= 2;
  if (a.dt == DT_BF16)
    return w == 1 ? launch_w<bf16_t, 1>(a, s) : w == 2 ? launch_w<bf16_t, 2>(a, s) : w == 4 ? launch_w<bf16_t, 4>(a, s) : launch_w<bf16_t, 8>(a, s);
  return w == 1 ? launch_w<float, 1>(a, s) : w == 2 ? launch_w<float, 2>(a, s) : w == 4 ? launch_w<float, 4>(a, s) : launch_w<float, 8>(a, s);
}

}  // namespace pf
