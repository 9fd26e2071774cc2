// Elements of a matrix in memory, of any type and at any address, and a tile's results on their way there.
#pragma once

#include "ob_mm.h"

namespace obm {

constexpr int BLOCK = 256;      // threads of the element-wise kernels

enum { F32 = 0, F16 = 1, BF16 = 2 };      // ob_dtype

typedef unsigned short v4h __attribute__((ext_vector_type(4)));
typedef float v4f_any __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned short v4h_any __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ float from_bits(unsigned short h, bool bf) {
  return bf ? __uint_as_float((unsigned)h << 16) : (float)__builtin_bit_cast(_Float16, h);
}
// to nearest, ties to even (a NaN stays one)
__device__ __forceinline__ unsigned short to_bits(float x, bool bf) {
  return bf ? __builtin_bit_cast(unsigned short, (__bf16)x) : __builtin_bit_cast(unsigned short, (_Float16)x);
}

// Four values in a row from p + at on, of which those from `left` on do not exist (and read as zeros).
__device__ __forceinline__ v4f load4(const void* p, int dtype, int64_t at, int left) {
  v4f v = {};
  if (left <= 0) return v;
  if (dtype == F32) {
    const float* const s = static_cast<const float*>(p) + at;
    if (left >= 4) return *reinterpret_cast<const v4f_any*>(s);
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < left) v[e] = s[e];
  } else {
    const unsigned short* const s = static_cast<const unsigned short*>(p) + at;
    v4h h = {};
    if (left >= 4) {
      h = *reinterpret_cast<const v4h_any*>(s);
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (e < left) h[e] = s[e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = from_bits(h[e], dtype == BF16);
  }
  return v;
}
__device__ __forceinline__ void store4(void* p, int dtype, int64_t at, int left, v4f v) {
  if (left <= 0) return;
  if (dtype == F32) {
    float* const s = static_cast<float*>(p) + at;
    if (left >= 4) {
      *reinterpret_cast<v4f_any*>(s) = v;
      return;
    }
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < left) s[e] = v[e];
  } else {
    unsigned short* const s = static_cast<unsigned short*>(p) + at;
    v4h h;
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = to_bits(v[e], dtype == BF16);
    if (left >= 4) {
      *reinterpret_cast<v4h_any*>(s) = h;
      return;
    }
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < left) s[e] = h[e];
  }
}

// store4 of binary32 values of which those before `from` belong to another tile
__device__ __forceinline__ void store_from(void* p, int64_t at, int left, int from, v4f v) {
  if (from <= 0) {
    store4(p, F32, at, left, v);
    return;
  }
#pragma unroll
  for (int e = 1; e < 4; ++e)
    if (e >= from && e < left) static_cast<float*>(p)[at + e] = v[e];
}

// A tile's results to `out` [rows, cols], rows ld elements apart, from its row r0 and column c0 on: 128 bytes of a row by eight lanes
// with 16-bit numbers, by sixteen (256 bytes) with binary32 ones.  Rows before row0 and columns before col0 are another
// tile's.  BF: the 16-bit type, if dtype is not F32.
template <class S, bool BF>
__device__ __forceinline__ void store_tile(const v4f (&acc)[S::FM][S::FN], uint16_t* lds, void* out, int dtype, int64_t ld, int r0, int c0, int rows,
                                           int cols, int row0, int col0) {
  using R = Results<S>;
  if (dtype == F32) {
    R::by_rows(acc, lds, [&](int r, int c, v4f v) {
      r += r0;
      c += c0;
      if (r >= row0 && r < rows && c + 3 >= col0) store_from(out, (int64_t)r * ld + c, cols - c, col0 - c, v);
    });
    return;
  }
  R::visit(acc, lds, [&](const float* own, int tr, int tc) {
    constexpr int EIGHTS = R::ROWS * R::WIDTH / 8, BATCH = EIGHTS / 64 < 4 ? EIGHTS / 64 : 4;
    const int lane = threadIdx.x & 63;
#pragma unroll 1
    for (int k0 = lane; k0 < EIGHTS; k0 += BATCH * 64) {
      v8s v[BATCH];
#pragma unroll
      for (int u = 0; u < BATCH; ++u) {
        const int k = k0 + u * 64;
        const float* const at = own + k / (R::WIDTH / 8) * R::STRIDE + k % (R::WIDTH / 8) * 8;
        const v4f lo = *in_lds<const v4f>(at), hi = *in_lds<const v4f>(at + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[u][e] = (short)to_bits(lo[e], BF);
          v[u][e + 4] = (short)to_bits(hi[e], BF);
        }
      }
#pragma unroll
      for (int u = 0; u < BATCH; ++u) {
        const int k = k0 + u * 64, r = r0 + tr + k / (R::WIDTH / 8), c = c0 + tc + k % (R::WIDTH / 8) * 8, left = cols - c;
        if (r < row0 || r >= rows || left <= 0 || c + 7 < col0) continue;
        uint16_t* const at = static_cast<uint16_t*>(out) + (int64_t)r * ld + c;
        if (left >= 8 && c >= col0) {
          *reinterpret_cast<v8s_any*>(at) = v[u];
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (e < left && c + e >= col0) at[e] = (uint16_t)v[u][e];
        }
      }
    }
  });
}

}  // namespace obm
