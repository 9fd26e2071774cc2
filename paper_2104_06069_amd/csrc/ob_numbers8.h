// Numbers of 8 bits with a scale for each block (include/ob_layer.h): the scale of a block and the bytes of its numbers.
//
// A scale is a power of two, so that a quotient is exact wherever it is not far below the format's smallest number, and is
// rounded once, by the conversion.
#pragma once

#include <type_traits>

#include "ob_elements.h"

namespace obl {

using namespace obm;

constexpr int BLOCK8 = 128;      // numbers of a block along a row
enum { E4M3 = 0, E5M2 = 1 };
typedef int v8i __attribute__((ext_vector_type(8)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v2i __attribute__((ext_vector_type(2)));
typedef unsigned v8u __attribute__((ext_vector_type(8)));
typedef unsigned short v8us __attribute__((ext_vector_type(8)));
typedef short v2s __attribute__((ext_vector_type(2)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef _Float16 v2hf __attribute__((ext_vector_type(2)));

// The byte of the scale of a block whose largest magnitude has these bits.  The largest numbers are 1.75 2^8 and 1.75 2^15: an amax
// of m 2^e needs 2^(e - 8) while m <= 1.75, and twice that above.
__device__ __forceinline__ int scale_byte(unsigned amax, int format) {
  if (amax >= 0x7f800000u) return 255;
  const int e = (int)((amax + 0x1fffffu) >> 23);
  return max(e - (format == E4M3 ? 8 : 15), 1);
}
// Eight bytes of a block of infinities or NaNs (byte 255) are NaNs, up to `left`, the others zeros
__device__ __forceinline__ v2i bytes_of_nans(int left) {
  const unsigned long long keep = left >= 8 ? ~0ull : left <= 0 ? 0 : ~0ull >> (64 - 8 * left);
  return v2i{(int)(0x7f7f7f7fu & (unsigned)keep), (int)(0x7f7f7f7fu & (unsigned)(keep >> 32))};
}

// Eight adjacent elements of one type as memory has them.  Those from `left` on do not exist and read as zeros.  PAST the caches: nothing
// of what is read stays there.
template <int DTYPE>
struct Raw8 {
  v8s h;
  template <bool PAST = false>
  __device__ __forceinline__ void load(const void* p, int64_t at, int left) {
    const uint16_t* const s = static_cast<const uint16_t*>(p) + at;
    h = v8s{};
    if (left >= 8) {
      if constexpr (PAST) h = __builtin_nontemporal_load(reinterpret_cast<const v8s_any*>(s));
      else h = *reinterpret_cast<const v8s_any*>(s);
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
  // Two adjacent ones over a power of two, to nearest, ties to even, as two bytes of `to`: the instruction's own division is exact for these types
  // and binary32 alike (found by trying all numbers of 16 bits that the quotient's format has room for)
  template <int FORMAT, bool HIGH>
  __device__ __forceinline__ v2s two(v2s to, int pair, float scale) const {
    const v2s w{h[2 * pair], h[2 * pair + 1]};
    if constexpr (DTYPE == BF16) {
      const auto b = __builtin_bit_cast(v2bf, w);
      return FORMAT == E4M3 ? __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(to, b, scale, HIGH) : __builtin_amdgcn_cvt_scalef32_pk_bf8_bf16(to, b, scale, HIGH);
    } else {
      const auto b = __builtin_bit_cast(v2hf, w);
      return FORMAT == E4M3 ? __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(to, b, scale, HIGH) : __builtin_amdgcn_cvt_scalef32_pk_bf8_f16(to, b, scale, HIGH);
    }
  }
  // Magnitudes, in bits that are ordered as they are; and as binary32's
  typedef v8us Magnitudes;
  __device__ __forceinline__ Magnitudes magnitudes() const { return __builtin_bit_cast(v8us, h) & (unsigned short)0x7fff; }
  __device__ static __forceinline__ unsigned of_binary32(unsigned short m) { return __float_as_uint(from_bits(m, DTYPE == BF16)); }
};
template <>
struct Raw8<F32> {
  v4f lo, hi;
  template <bool PAST = false>
  __device__ __forceinline__ void load(const void* p, int64_t at, int left) {
    if (PAST && left >= 8) {
      lo = __builtin_nontemporal_load(reinterpret_cast<const v4f_any*>(static_cast<const float*>(p) + at));
      hi = __builtin_nontemporal_load(reinterpret_cast<const v4f_any*>(static_cast<const float*>(p) + at + 4));
      return;
    }
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
  template <int FORMAT, bool HIGH>
  __device__ __forceinline__ v2s two(v2s to, int pair, float scale) const {
    const v4f v = pair < 2 ? lo : hi;
    const float a = v[pair % 2 * 2], b = v[pair % 2 * 2 + 1];
    return FORMAT == E4M3 ? __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(to, a, b, scale, HIGH) : __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(to, a, b, scale, HIGH);
  }
  typedef v8u Magnitudes;
  __device__ __forceinline__ Magnitudes magnitudes() const {
    return __builtin_bit_cast(v8u, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7)) & 0x7fffffffu;
  }
  __device__ static __forceinline__ unsigned of_binary32(unsigned m) { return m; }
};
template <class RAW, int FORMAT>
__device__ __forceinline__ v2i bytes8(const RAW& r, float scale) {
  const v2s none{};
  return v2i{__builtin_bit_cast(int, r.template two<FORMAT, true>(r.template two<FORMAT, false>(none, 0, scale), 1, scale)),
             __builtin_bit_cast(int, r.template two<FORMAT, true>(r.template two<FORMAT, false>(none, 2, scale), 3, scale))};
}
// Eight numbers over the scale of this byte; those from `left` on are zeros
template <class RAW>
__device__ __forceinline__ v2i bytes8(const RAW& r, int byte, int format, int left) {
  const float scale = __uint_as_float((unsigned)byte << 23);
  v2i q = format == E4M3 ? bytes8<RAW, E4M3>(r, scale) : bytes8<RAW, E5M2>(r, scale);
  if (byte == 255) q = bytes_of_nans(left);
  return q;
}
template <class V>
__device__ __forceinline__ unsigned highest(V m) {      // of eight magnitudes
  const auto four = __builtin_elementwise_max(__builtin_shufflevector(m, m, 0, 1, 2, 3), __builtin_shufflevector(m, m, 4, 5, 6, 7));
  const auto two = __builtin_elementwise_max(__builtin_shufflevector(four, four, 0, 1), __builtin_shufflevector(four, four, 2, 3));
  return max((unsigned)two[0], (unsigned)two[1]);
}
// The largest of sixteen adjacent lanes', for all of them: the lanes' values turned by 8, 4, 2 and 1
template <class V>
__device__ __forceinline__ V highest_of_16(V m) {
  constexpr int WORDS = sizeof(V) / 4;
  struct Words {
    int w[WORDS];
  };
  const auto turned = [](V v, auto by) {
    auto w = __builtin_bit_cast(Words, v);
#pragma unroll
    for (int k = 0; k < WORDS; ++k) w.w[k] = __builtin_amdgcn_update_dpp(0, w.w[k], 0x120 + decltype(by)::value, 0xf, 0xf, true);
    return __builtin_bit_cast(V, w);
  };
  m = __builtin_elementwise_max(m, turned(m, std::integral_constant<int, 8>{}));
  m = __builtin_elementwise_max(m, turned(m, std::integral_constant<int, 4>{}));
  m = __builtin_elementwise_max(m, turned(m, std::integral_constant<int, 2>{}));
  return __builtin_elementwise_max(m, turned(m, std::integral_constant<int, 1>{}));
}
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
