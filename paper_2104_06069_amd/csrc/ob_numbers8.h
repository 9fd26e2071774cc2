// Numbers of 8 bits with a scale for each block (include/ob_layer.h): the scale of a block and the bytes of its numbers.
//
// A scale is a power of two, so that a quotient is exact wherever it is not far below the format's smallest number, and is
// rounded once, by the conversion.
#pragma once

#include "ob_elements.h"

namespace obl {

using namespace obm;

constexpr int BLOCK8 = 128;      // numbers of a block along a row
enum { E4M3 = 0, E5M2 = 1 };
typedef int v8i __attribute__((ext_vector_type(8)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v2i __attribute__((ext_vector_type(2)));

__device__ __forceinline__ unsigned magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }      // (a NaN's is above an infinity's)

// The byte of the scale of a block whose largest magnitude has these bits.  The largest numbers are 1.75 2^8 and 1.75 2^15: an amax
// of m 2^e needs 2^(e - 8) while m <= 1.75, and twice that above.
__device__ __forceinline__ int scale_byte(unsigned amax, int format) {
  if (amax >= 0x7f800000u) return 255;
  const int e = (int)((amax + 0x1fffffu) >> 23);
  return max(e - (format == E4M3 ? 8 : 15), 1);
}
// One over the scale: 2^(127 - byte), NaN for 255.  (The bytes of finite blocks are 1 .. 247: the result is a normal number.)
__device__ __forceinline__ float inverse_scale(int byte) { return byte == 255 ? __uint_as_float(0x7fc00000u) : __uint_as_float((unsigned)(254 - byte) << 23); }

// Four bytes of four values times `inv`, to nearest, ties to even
__device__ __forceinline__ int bytes4(float a, float b, float c, float d, float inv, int format) {
  a *= inv;
  b *= inv;
  c *= inv;
  d *= inv;
  if (format == E4M3) return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
  return __builtin_amdgcn_cvt_pk_bf8_f32(c, d, __builtin_amdgcn_cvt_pk_bf8_f32(a, b, 0, false), true);
}
__device__ __forceinline__ v2i bytes8(const float (&v)[8], float inv, int format) {
  v2i r;
  r.x = bytes4(v[0], v[1], v[2], v[3], inv, format);
  r.y = bytes4(v[4], v[5], v[6], v[7], inv, format);
  return r;
}

// Eight adjacent elements of one type as memory has them.  Those from `left` on do not exist and read as zeros.
template <int DTYPE>
struct Raw8 {
  v8s h;
  __device__ __forceinline__ void load(const void* p, int64_t at, int left) {
    const uint16_t* const s = static_cast<const uint16_t*>(p) + at;
    h = v8s{};
    if (left >= 8) {
      h = *reinterpret_cast<const v8s_any*>(s);
    } else {
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if (e < left) h[e] = (short)s[e];
    }
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = from_bits((unsigned short)h[e], DTYPE == BF16);
  }
  __device__ __forceinline__ void forget() { asm volatile("" : "+v"(h)); }      // (what was made of it before is made again)
};
template <>
struct Raw8<F32> {
  v4f lo, hi;
  __device__ __forceinline__ void load(const void* p, int64_t at, int left) {
    lo = load4(p, F32, at, left);
    hi = load4(p, F32, at + 4, left - 4);
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = lo[e];
      v[e + 4] = hi[e];
    }
  }
  __device__ __forceinline__ void forget() {}
};
template <int DTYPE>
__device__ __forceinline__ void load8(const void* p, int64_t at, int left, float (&v)[8]) {
  Raw8<DTYPE> r;
  r.load(p, at, left);
  r.values(v);
}
template <int DTYPE>
__device__ __forceinline__ void store8(void* p, int64_t at, int left, const float (&v)[8]) {
  if constexpr (DTYPE == F32) {
    store4(p, F32, at, left, v4f{v[0], v[1], v[2], v[3]});
    store4(p, F32, at + 4, left - 4, v4f{v[4], v[5], v[6], v[7]});
  } else {
    uint16_t* const s = static_cast<uint16_t*>(p) + at;
    v8s h;
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = (short)to_bits(v[e], DTYPE == BF16);
    if (left >= 8) {
      *reinterpret_cast<v8s_any*>(s) = h;
    } else {
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if (e < left) s[e] = (uint16_t)h[e];
    }
  }
}
__device__ __forceinline__ void load8_any(const void* p, int dtype, int64_t at, int left, float (&v)[8]) {
  if (dtype == F32) load8<F32>(p, at, left, v);
  else if (dtype == F16) load8<F16>(p, at, left, v);
  else load8<BF16>(p, at, left, v);
}
// v as memory holds it after store8
template <int DTYPE>
__device__ __forceinline__ float as_stored(float x) {
  return DTYPE == F32 ? x : from_bits(to_bits(x, DTYPE == BF16), DTYPE == BF16);
}

}  // namespace obl
