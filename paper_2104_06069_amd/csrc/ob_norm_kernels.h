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

template <class V>
__device__ __forceinline__ V wave_sum(V v) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d);
  return v;
}
// The sum over the T threads of a row; `part` holds a place for each wavefront of the workgroup, not in use by another sum.
template <int T, class V>
__device__ __forceinline__ V row_sum(V v, V* part) {
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

// Whether a row's mean of squares, with eps, lies where binary32 has lost nothing of it: no square above its largest number, and none
// that counts below its smallest
__device__ __forceinline__ bool in_range(float mean) { return mean >= 0x1p-100f && mean <= 0x1.fffffep127f; }

template <int X, int H, int T, int C>
__global__ __launch_bounds__(T < 256 ? 256 : T) void k_norm_forward(NormArgs p) {
  constexpr int NT = T < 256 ? 256 : T;
  __shared__ float part[NT / 64];
  __shared__ double part64[NT / 64];
  const int t = threadIdx.x % T;
  const int64_t row = (int64_t)blockIdx.x * (NT / T) + threadIdx.x / T;
  const bool there = row < p.rows;
  if (T <= 64 && !there) return;
  // Every load is under way before the first sum; the weights too, where there are registers for them.
  constexpr bool EARLY = C <= 2;
  Raw8<X> x[C];
  Raw8<H> r[C];
  float w[EARLY ? C : 1][8], h[C][8], sum = 0;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int at = (c * T + t) * 8, left = there ? p.n - at : 0;
    x[c].load(p.x, row * p.ldx + at, left);
    if (p.residual) r[c].load(p.residual, row * p.ldr + at, left);
  }
  if constexpr (EARLY) {
    if (p.weight) {
#pragma unroll
      for (int c = 0; c < C; ++c) load8_any(p.weight, p.weight_dtype, (c * T + t) * 8, p.n - (c * T + t) * 8, w[c]);
    }
  }
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int at = (c * T + t) * 8, left = there ? p.n - at : 0;
    x[c].values(h[c]);
    if (p.residual) {
      float v[8];
      r[c].values(v);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[c][e] = as_stored<H>(h[c][e] + v[e]);
      if (left > 0) store8<H>(p.h, row * p.ldh + at, left, h[c]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += h[c][e] * h[c][e];
  }
  sum = row_sum<T>(sum, part);
  const float mean = sum / (float)p.n + p.eps;
  float rstd = 1.0f / sqrtf(mean);
  bool again = !in_range(mean);
  if constexpr (T > 64 && NT > T) {      // rows of a workgroup go to the same barriers
#pragma unroll
    for (int r = 0; r < NT / T; ++r) {
      float s = 0;
#pragma unroll
      for (int w = 0; w < T / 64; ++w) s += part[r * (T / 64) + w];
      again |= !in_range(s / (float)p.n + p.eps);
    }
  }
  if (again) {      // squares of binary32 numbers are exact in binary64, and their sums are in its range
    double s = 0;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fma((double)h[c][e], (double)h[c][e], s);
    s = row_sum<T>(s, part64);
    if (!in_range(mean)) rstd = (float)(1.0 / sqrt(s / (double)p.n + (double)p.eps));
  }
  if (!there) return;
  if (t == 0 && p.rstd) p.rstd[row] = rstd;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int at = (c * T + t) * 8, left = p.n - at;
    if constexpr (!EARLY) {
      if (p.weight) load8_any(p.weight, p.weight_dtype, at, left, w[0]);
    }
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = h[c][e] * rstd;
    if (p.weight) {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = y[e] * w[EARLY ? c : 0][e];
    }
    if (p.y && left > 0) store8<X>(p.y, row * p.ldy + at, left, y);
    if (p.data) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e >= left) y[e] = 0;      // (0 times an rstd that is not finite)
      const Raw8<F32> raw{v4f{y[0], y[1], y[2], y[3]}, v4f{y[4], y[5], y[6], y[7]}};
      const int byte = scale_byte(highest_of_16(highest(raw.magnitudes())), p.format), padded = (p.n + BLOCK8 - 1) / BLOCK8 * BLOCK8;
      const v2i q = bytes8(raw, byte, p.format, left);      // (behind the row's end zeros, in a block of NaNs too)
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
  __shared__ float sums[SETS > 1 ? T * 8 : 1];
  const int t = threadIdx.x % T, set = threadIdx.x / T;
  float dw[C][8] = {};
  int turn = 0;
  for (int64_t first = (int64_t)blockIdx.x * SETS; first < p.rows; first += (int64_t)gridDim.x * SETS, turn ^= 1) {
    const int64_t row = first + set;
    const bool there = row < p.rows;
    const float rstd = there ? p.rstd[row] : 0.0f;
    // (Across the sum the row stays as memory has it, and is unpacked twice: half the registers of its values.)
    Raw8<X> dy[C];
    Raw8<H> h[C], dres[C];
    float dot = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int at = (c * T + t) * 8, left = there ? p.n - at : 0;
      dy[c].load(p.dy, row * p.lddy + at, left);
      h[c].load(p.h, row * p.ldh + at, left);
    }
    if (p.dres) {
#pragma unroll
      for (int c = 0; c < C; ++c) dres[c].load(p.dres, row * p.lddres + (c * T + t) * 8, there ? p.n - (c * T + t) * 8 : 0);
    }
    const auto unpack = [&](int c, float (&g)[8], float (&xhat)[8]) {
      dy[c].values(g);
      h[c].values(xhat);
#pragma unroll
      for (int e = 0; e < 8; ++e) xhat[e] = e < p.n - (c * T + t) * 8 ? xhat[e] * rstd : 0.0f;      // (rstd may be no finite number)
    };
    const void* weight = p.weight;
    const auto weigh = [&](int c, float (&g)[8]) {
      float w[8];
      if (!weight) return;
      load8_any(weight, p.weight_dtype, (c * T + t) * 8, p.n - (c * T + t) * 8, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) g[e] = g[e] * w[e];
    };
    asm volatile("" : "+s"(weight));      // (read for each row, from the nearest cache, and not held in registers)
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float g[8], xhat[8];
      unpack(c, g, xhat);
#pragma unroll
      for (int e = 0; e < 8; ++e) dw[c][e] += g[e] * xhat[e];
      weigh(c, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) dot += g[e] * xhat[e];
    }
    if (!p.dh) continue;      // (the same for all of them)
    dot = row_sum<T>(dot, part[turn]) / (float)p.n;
    if (!there) continue;
    asm volatile("" : "+s"(weight));
#pragma unroll
    for (int c = 0; c < C; ++c) {
      dy[c].forget();
      h[c].forget();
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int at = (c * T + t) * 8, left = p.n - at;
      if (left <= 0) continue;
      float g[8], xhat[8], r[8];
      unpack(c, g, xhat);
      weigh(c, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) g[e] = rstd * (g[e] - xhat[e] * dot);
      if (p.dres) {
        dres[c].values(r);
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] += r[e];
      }
      store8<H>(p.dh, row * p.lddh + at, left, g);
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

// dweight[j] = sum over the workgroups, in their order: 64 columns a workgroup, SHARES shares of the sums, then those.
constexpr int SHARES = 16;
__global__ __launch_bounds__(SHARES * 64) void k_norm_join(const float* partial, int parts, int n, int accumulate, float* dweight) {
  __shared__ float share[SHARES][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x / 64, j = blockIdx.x * 64 + lane;
  float s = 0;
  const int each = (parts + SHARES - 1) / SHARES, end = min(parts, (w + 1) * each);
  if (j < n) {
#pragma unroll 8
    for (int g = w * each; g < end; ++g) s += partial[(int64_t)g * n + j];
  }
  share[w][lane] = s;
  __syncthreads();
  if (w == 0 && j < n) {
    s = share[0][lane];
#pragma unroll
    for (int k = 1; k < SHARES; ++k) s += share[k][lane];
    dweight[j] = accumulate ? dweight[j] + s : s;
  }
}

}  // namespace obl
