// Kernels of the root-mean-square norm (include/ob_layer.h).  Included by ob_norm.hip only.
//
// T threads hold a row in registers, C pieces of eight adjacent numbers each (piece c of thread t begins at number (c T + t) 8),
// so that every operand is read once and every result written once; the sums over a row are a tree over the threads.  128
// numbers of a block are those of sixteen adjacent lanes.
#pragma once

#include "ob_numbers8.h"

namespace obl {

struct NormArgs {
  const void *x, *residual, *weight;
  void *h, *y;
  uint8_t *data, *scales;
  float* rstd;
  int64_t ldx, ldr, ldh, ldy, ld, ld_scales;
  int rows, n, weight_dtype, format;
  float eps;
};

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d);
  return v;
}
// The sum over the T threads of a row; `part` holds a place for each wavefront of the workgroup, not in use by another sum.
template <int T>
__device__ __forceinline__ float row_sum(float v, float* part) {
  v = wave_sum(v);
  if constexpr (T > 64) {
    const int wave = threadIdx.x / 64, first = threadIdx.x / T * (T / 64);
    if ((threadIdx.x & 63) == 0) part[wave] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < T / 64; ++w) v += part[first + w];
  }
  return v;
}

template <int X, int H, int T, int C>
__global__ __launch_bounds__(T < 256 ? 256 : T) void k_norm_forward(NormArgs p) {
  constexpr int NT = T < 256 ? 256 : T;
  __shared__ float part[NT / 64];
  const int t = threadIdx.x % T;
  const int64_t row = (int64_t)blockIdx.x * (NT / T) + threadIdx.x / T;
  const bool there = row < p.rows;
  if (T <= 64 && !there) return;
  float h[C][8], sum = 0;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int at = (c * T + t) * 8, left = there ? p.n - at : 0;
    load8<X>(p.x, row * p.ldx + at, left, h[c]);
    if (p.residual) {
      float r[8];
      load8<H>(p.residual, row * p.ldr + at, left, r);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[c][e] = as_stored<H>(h[c][e] + r[e]);
      if (left > 0) store8<H>(p.h, row * p.ldh + at, left, h[c]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += h[c][e] * h[c][e];
  }
  sum = row_sum<T>(sum, part);
  if (!there) return;
  const float rstd = 1.0f / sqrtf(sum / (float)p.n + p.eps);
  if (t == 0 && p.rstd) p.rstd[row] = rstd;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int at = (c * T + t) * 8, left = p.n - at;
    float w[8];
    if (p.weight) load8_any(p.weight, p.weight_dtype, at, left, w);
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = h[c][e] * rstd;
    if (p.weight) {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = y[e] * w[e];
    }
    if (p.y && left > 0) store8<X>(p.y, row * p.ldy + at, left, y);
    if (p.data) {
      unsigned most = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (e >= left) y[e] = 0;      // (0 times an rstd that is not finite)
        most = max(most, magnitude(y[e]));
      }
#pragma unroll
      for (int d = 8; d >= 1; d >>= 1) most = max(most, (unsigned)__shfl_xor((int)most, d));
      const int byte = scale_byte(most, p.format), padded = (p.n + BLOCK8 - 1) / BLOCK8 * BLOCK8;
      v2i q = bytes8(y, inverse_scale(byte), p.format);
      if (left < 8) {      // behind the row's end: zeros in a block of NaNs too
        unsigned long long keep = left <= 0 ? 0 : ~0ull >> (64 - 8 * left);
        q.x &= (int)(unsigned)keep;
        q.y &= (int)(unsigned)(keep >> 32);
      }
      if (at < padded) *reinterpret_cast<v2i*>(p.data + row * p.ld + at) = q;
      if (at % BLOCK8 == 0 && left > 0) p.scales[row * p.ld_scales + at / BLOCK8] = (uint8_t)byte;
    }
  }
}

struct NormGradArgs {
  const void *dy, *h, *weight, *dres;
  const float* rstd;
  void* dh;
  float *dweight, *partial;      // partial [workgroups, n], unless there is one
  int64_t lddy, ldh, lddres, lddh;
  int rows, n, weight_dtype, accumulate;
};

// Each workgroup takes every gridDim.x-th set of rows and sums dy xhat over them in registers; k_norm_join adds the workgroups' sums.
template <int T>
constexpr int norm_grad_threads() { return T < 512 ? 512 : T; }
template <int X, int H, int T, int C>
__global__ __launch_bounds__(norm_grad_threads<T>()) void k_norm_backward(NormGradArgs p) {
  constexpr int NT = norm_grad_threads<T>(), SETS = NT / T;      // rows at a time
  __shared__ float part[2][NT / 64];
  __shared__ float sums[T * 8];
  const int t = threadIdx.x % T, set = threadIdx.x / T;
  float dw[C][8] = {};
  int turn = 0;
  for (int64_t first = (int64_t)blockIdx.x * SETS; first < p.rows; first += (int64_t)gridDim.x * SETS, turn ^= 1) {
    const int64_t row = first + set;
    const bool there = row < p.rows;
    const float rstd = there ? p.rstd[row] : 0.0f;
    float g[C][8], xhat[C][8], dot = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int at = (c * T + t) * 8, left = there ? p.n - at : 0;
      load8<X>(p.dy, row * p.lddy + at, left, g[c]);
      load8<H>(p.h, row * p.ldh + at, left, xhat[c]);
      float w[8];
      if (p.weight) load8_any(p.weight, p.weight_dtype, at, p.n - at, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        xhat[c][e] = e < left ? xhat[c][e] * rstd : 0.0f;      // (rstd may be no finite number)
        dw[c][e] += g[c][e] * xhat[c][e];
        if (p.weight) g[c][e] = g[c][e] * w[e];
        dot += g[c][e] * xhat[c][e];
      }
    }
    if (!p.dh) continue;      // (the same for all of them)
    dot = row_sum<T>(dot, part[turn]) / (float)p.n;
    if (!there) continue;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int at = (c * T + t) * 8, left = p.n - at;
      if (left <= 0) continue;
      float d[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) d[e] = rstd * (g[c][e] - xhat[c][e] * dot);
      if (p.dres) {
        float r[8];
        load8<H>(p.dres, row * p.lddres + at, left, r);
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] += r[e];
      }
      store8<H>(p.dh, row * p.lddh + at, left, d);
    }
  }
  if (!p.dweight) return;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int at = (c * T + t) * 8, left = p.n - at;
    if constexpr (SETS > 1) {      // set by set into the first one's
#pragma unroll 1
      for (int s = SETS - 1; s >= 1; --s) {
        __syncthreads();
        if (set == s) {
#pragma unroll
          for (int e = 0; e < 8; ++e) sums[t * 8 + e] = dw[c][e];
        }
        __syncthreads();
        if (set == s - 1) {
#pragma unroll
          for (int e = 0; e < 8; ++e) dw[c][e] += sums[t * 8 + e];
        }
      }
    }
    if (set == 0 && left > 0) {
      if (gridDim.x > 1) {
        store8<F32>(p.partial + (int64_t)blockIdx.x * p.n, at, left, dw[c]);
      } else {
        float old[8] = {};
        if (p.accumulate) load8<F32>(p.dweight, at, left, old);
#pragma unroll
        for (int e = 0; e < 8; ++e) old[e] += dw[c][e];
        store8<F32>(p.dweight, at, left, old);
      }
    }
  }
}

// dweight[j] = sum over the workgroups, in their order: 64 columns a workgroup, four shares of the sums, then those four.
__global__ __launch_bounds__(256) void k_norm_join(const float* partial, int parts, int n, int accumulate, float* dweight) {
  __shared__ float share[4][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x / 64, j = blockIdx.x * 64 + lane;
  float s = 0;
  const int each = (parts + 3) / 4, end = min(parts, (w + 1) * each);
  if (j < n)
    for (int g = w * each; g < end; ++g) s += partial[(int64_t)g * n + j];
  share[w][lane] = s;
  __syncthreads();
  if (w == 0 && j < n) {
    s = ((share[0][lane] + share[1][lane]) + share[2][lane]) + share[3][lane];
    dweight[j] = accumulate ? dweight[j] + s : s;
  }
}

}  // namespace obl
