// Kernels of the gradient's norm and its clipping (include/ob_layer.h).  Included by ob_clip.hip only.
//
// Squares are summed in binary64, in which the square of a binary32 number is exact, so that no gradient over- or underflows on
// its way into the norm.  A tensor is cut into segments, a workgroup each; the sums over a tensor's segments and over the tensors have
// one order.
#pragma once

#include "ob_numbers8.h"

namespace obl {

struct Segment {
  int64_t at;
  int32_t len, layer;
};

// 16 bytes of elements, read past the caches, which hold nothing of a large gradient until it comes around again (302 M binary32 numbers: norm 208
// us without, 187 with; clipped 642 and 591)
template <int DTYPE>
struct Piece {
  static constexpr int N = DTYPE == F32 ? 4 : 8;
  __device__ static __forceinline__ void load(const void* p, int64_t at, int64_t left, float (&v)[N]) {
    if constexpr (DTYPE == F32) {
      const v4f w = left >= 4 ? __builtin_nontemporal_load(reinterpret_cast<const v4f_any*>(static_cast<const float*>(p) + at)) : load4(p, F32, at, (int)left);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = w[e];
    } else if (left >= 8) {
      const v8s h = __builtin_nontemporal_load(reinterpret_cast<const v8s_any*>(static_cast<const uint16_t*>(p) + at));
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = from_bits((unsigned short)h[e], DTYPE == BF16);
    } else {
      load8<DTYPE>(p, at, (int)left, v);
    }
  }
};

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d);
  return v;
}
// Over the four wavefronts of a workgroup, for all of its threads
__device__ __forceinline__ double group_sum(double v) {
  __shared__ double part[4];
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  return (part[0] + part[1]) + (part[2] + part[3]);
}

template <int DTYPE>
__global__ __launch_bounds__(256) void k_clip_squares(const Segment* segments, const void* grad, double* sums) {
  using P = Piece<DTYPE>;
  const Segment s = segments[blockIdx.x];
  double sum[P::N] = {};
  constexpr int AHEAD = 4;
  for (int at = threadIdx.x * P::N; at < s.len; at += AHEAD * 256 * P::N) {
    float v[AHEAD][P::N];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) P::load(grad, s.at + at + u * 256 * P::N, s.len - at - u * 256 * P::N, v[u]);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
#pragma unroll
      for (int e = 0; e < P::N; ++e) sum[e] = fma((double)v[u][e], (double)v[u][e], sum[e]);
  }
#pragma unroll
  for (int e = 1; e < P::N; ++e) sum[0] += sum[e];
  const double all = group_sum(sum[0]);
  if (threadIdx.x == 0) sums[blockIdx.x] = all;
}

struct ClipArgs {
  const double* sums;          // of the segments
  const int* first;            // [layers + 1]: a tensor's first segment
  double* layer_sums;
  unsigned* ticket;            // 0 between calls
  float *norm, *layer_norms;   // layer_norms: or NULL
  int layers, segments;
  float grad_scale, eps, max_norm;
};

// sum over a tensor's segments, by a wavefront
__device__ __forceinline__ double layer_sum(const ClipArgs& p, int l) {
  double v = 0;
  const int end = p.first[l + 1];
  for (int s = p.first[l] + (threadIdx.x & 63); s < end; s += 64) v += p.sums[s];
  return wave_sum(v);
}
__device__ __forceinline__ float norm_of(double squares, float scale) { return (float)((double)scale * sqrt(squares)); }

// A wavefront a tensor; the workgroup that is done last adds up the tensors.
__global__ __launch_bounds__(256) void k_clip_norm(ClipArgs p) {
  __shared__ unsigned order;
  const int l = blockIdx.x * 4 + threadIdx.x / 64;
  if (l < p.layers) {
    const double v = layer_sum(p, l);
    if ((threadIdx.x & 63) == 0) {
      __hip_atomic_store(&p.layer_sums[l], v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (p.layer_norms) p.layer_norms[l] = norm_of(v, p.grad_scale);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // (there before the arrival: thread 0's fence waits for its own wavefront's stores alone)
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    order = __hip_atomic_fetch_add(p.ticket, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (order != gridDim.x - 1) return;
  __threadfence();
  double v = 0;
  for (int i = threadIdx.x; i < p.layers; i += 256) v += __hip_atomic_load(&p.layer_sums[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  v = group_sum(v);
  if (threadIdx.x == 0) {
    *p.norm = norm_of(v, p.grad_scale);
    __hip_atomic_store(p.ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
}

struct ClipApplyArgs {
  ClipArgs norm;
  const void* grad;
  void* out;
  int64_t n;
  bool apply, in_place;
};

template <int IN, int OUT, bool NORM>
__global__ __launch_bounds__(256) void k_clip_apply(ClipApplyArgs p) {
  using P = Piece<IN>;
  constexpr int EACH = 4, SPAN = EACH * 256 * P::N;
  const ClipArgs& c = p.norm;
  float norm;
  if constexpr (NORM) {      // few segments: every workgroup adds them up itself, and one launch less
    double v = 0;
    for (int i = threadIdx.x; i < c.segments; i += 256) v += c.sums[i];
    norm = norm_of(group_sum(v), c.grad_scale);
    if (blockIdx.x == 0 && threadIdx.x == 0) *c.norm = norm;
    if (c.layer_norms) {
      for (int l = blockIdx.x * 4 + threadIdx.x / 64; l < c.layers; l += gridDim.x * 4) {
        const double s = layer_sum(c, l);
        if ((threadIdx.x & 63) == 0) c.layer_norms[l] = norm_of(s, c.grad_scale);
      }
    }
    if (!p.apply) return;
  } else {
    norm = *c.norm;
  }
  const float most = norm + c.eps;
  const float f = c.grad_scale * (most <= c.max_norm ? 1.0f : c.max_norm / most);
  if (p.in_place && f == 1.0f) return;
  // (the end first: it was read last, and what of it is still in the memory-side cache comes from there)
  const int64_t at0 = (int64_t)(gridDim.x - 1 - blockIdx.x) * SPAN + threadIdx.x * P::N;
  float v[EACH][P::N];
#pragma unroll
  for (int u = 0; u < EACH; ++u) P::load(p.grad, at0 + u * 256 * P::N, p.n - at0 - u * 256 * P::N, v[u]);
#pragma unroll
  for (int u = 0; u < EACH; ++u) {
    const int64_t at = at0 + u * 256 * P::N;
    const int left = (int)min(p.n - at, (int64_t)P::N);
    if (left <= 0) continue;
#pragma unroll
    for (int e = 0; e < P::N; ++e) v[u][e] *= f;
    if constexpr (P::N == 8) {
      store8<OUT>(p.out, at, left, v[u]);
    } else {
      store4(p.out, OUT, at, left, v4f{v[u][0], v[u][1], v[u][2], v[u][3]});
    }
  }
}

}  // namespace obl
