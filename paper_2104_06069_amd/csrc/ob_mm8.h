// One workgroup's tile of C = A B^T with operands of 8 bits and a scale for each 128 columns of K, summed in binary32 on the
// matrix cores (gfx950), in one of two ways:
//   8-bit instructions, which take 128 columns at once and apply both operands' scales, powers of two, as they multiply: 4.7
//   PFLOP/s.  They cut each of eight adjacent products off 13 bits below the largest power of two among them before they sum them in
//   binary32, which makes 1.5e-5 (2-norm, normal numbers), whatever K is: far below the rounding of a 16-bit result.
//   WIDE, for binary32 results: operands made bfloat16 in registers, scales applied, both exactly, and the instructions for those, which
//   lose nothing before binary32 (7e-8 at K = 8192): half the rate.
//
// An operand's rows are K bytes, K a multiple of 128 and zeros behind the matrix, so that a slab of 128 columns is always whole.  In
// LDS it lies as a slab of 64 16-bit numbers does (Slab, ob_mm.h): what a lane gets are pieces q and q + 4 of its row in place of 2 q
// and 2 q + 1, of both operands alike, and of one block.  Beside a slab lie the scales of its rows, four bytes each, for the four
// slabs of a group.
#pragma once

#include <type_traits>

#include "ob_mm.h"
#include "ob_numbers8.h"

namespace obl {

struct Operand8 {
  const uint8_t *p, *scales;
  int64_t ld, ld_scales;
  int rows, shift;      // rows >= 1; row r has the scales of scale row r >> shift
};

// B's numbers are e4m3
template <int FORMAT>
__device__ __forceinline__ v4f mma8(v8i b, int scale_b, v8i a, int scale_a, v4f c) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, c, 0, FORMAT == E4M3 ? 0 : 1, 0, scale_b, 0, scale_a);
}

// Eight of a lane's bytes times the scale, as bfloat16: exact
template <int FORMAT>
__device__ __forceinline__ v8s widened(int lo, int hi, float scale) {
  const auto two = [&](int v, auto high) {
    if constexpr (FORMAT == E4M3) return __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, scale, decltype(high)::value));
    else return __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(v, scale, decltype(high)::value));
  };
  const std::false_type low;
  const std::true_type high;
  return __builtin_bit_cast(v8s, v4i{two(lo, low), two(lo, high), two(hi, low), two(hi, high)});
}
__device__ __forceinline__ float scale_value(int byte) { return __uint_as_float((unsigned)byte << 23); }      // (255: NaNs in the numbers themselves)

template <class S, int FORMAT, bool WIDE>
struct Product8 {
  static constexpr int BM = S::BM, BN = S::BN, BK = 64, FM = S::FM, FN = S::FN;      // (BK in pairs of bytes)
  static_assert(S::BK == BK && S::TEAMS == 1, "slabs of a block");
  using A = Slab<KC, BM, BK, S::NT>;
  using B = Slab<KC, BN, BK, S::NT>;
  static constexpr int SCALE_WAVES = (BM + BN) / 64, SCALES = (BM + BN) * BK;      // where a slab's scales begin
  static_assert(SCALE_WAVES <= S::WAVES, "a row's scales for each lane");
  static constexpr int STAGE = (BM + BN) * (BK + 2);
  static constexpr int LDS_BYTES = S::STAGES * STAGE * 2 > Results<S>::LDS_BYTES ? S::STAGES * STAGE * 2 : Results<S>::LDS_BYTES;
  typedef v4f Acc[FM][FN];

  // Slabs t0 .. t0 + n - 1 of K.  The layout of acc is Product's.
  __device__ static void run(const Operand8& oa, const Operand8& ob, int r0, int c0, int t0, int n, uint16_t* lds, Acc& acc) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / S::WN, wn = wave % S::WN;
    const Operand a{reinterpret_cast<const uint16_t*>(oa.p), 0, oa.ld / 2, oa.rows, true};
    const Operand b{reinterpret_cast<const uint16_t*>(ob.p), 0, ob.ld / 2, ob.rows, true};
    A sa;
    B sb;
    sa.init(a, r0, tid);
    sb.init(b, c0, tid);
    const Operand8& own = wave < BM / 64 ? oa : ob;
    const int of = wave < BM / 64 ? r0 + tid : c0 + tid - BM;
    const uint8_t* const scales = own.scales + (int64_t)(min(of, own.rows - 1) >> own.shift) * own.ld_scales;
    const auto load = [&](int t) {
      uint16_t* const s = lds + t % S::STAGES * STAGE;
      sa.load(a, 0, r0, (t0 + t) * BK, s, wave);
      sb.load(b, 0, c0, (t0 + t) * BK, s + BM * BK, wave);
      if (wave < SCALE_WAVES)
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(scales + (t0 + t) / 4 * 4), in_lds<void>(s + SCALES + wave * 128), 4, 0, 0);
    };
    const auto fragment = [&](const uint16_t* s, int row) {
      const v8s lo = A::fragment(s, row, 0, lane), hi = A::fragment(s, row, 1, lane);      // (the same for B: it goes by BK alone)
      return __builtin_bit_cast(v8i, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 14, 15));
    };
    const auto scale = [&](const uint16_t* s, int row, int t) {
      return (int)*in_lds<const uint8_t>(reinterpret_cast<const uint8_t*>(s + SCALES) + (row + (lane & 15)) * 4 + ((t0 + t) & 3));
    };
    const auto read_a = [&](const uint16_t* s, int i, int t, v8i& f, int& e) {
      const int row = wm * (BM / S::WM) + i * 16;
      f = fragment(s, row);
      e = scale(s, row, t);
    };
    const auto read_b = [&](const uint16_t* s, int j, int t, v8i& f, int& e) {
      const int row = wn * (BN / S::WN) + j * 16;
      f = fragment(s + BM * BK, row);
      e = scale(s, BM + row, t);
    };
    straight(n, wave, lds, load, read_a, read_b, acc);
  }

 private:
  // Rows of fragments I0 .. I0 + COUNT - 1 of acc
  template <int I0, int COUNT>
  __device__ static __forceinline__ void multiply(const v8i (&fa)[COUNT], const int (&ea)[COUNT], const v8i (&fb)[FN], const int (&eb)[FN], Acc& acc) {
    if constexpr (!WIDE) {
#pragma unroll
      for (int i = 0; i < COUNT; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[I0 + i][j] = mma8<FORMAT>(fb[j], eb[j], fa[i], ea[i], acc[I0 + i][j]);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        v8s wb[FN];
#pragma unroll
        for (int j = 0; j < FN; ++j) wb[j] = widened<E4M3>(fb[j][2 * k], fb[j][2 * k + 1], scale_value(eb[j]));
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
          const v8s wa = widened<FORMAT>(fa[i][2 * k], fa[i][2 * k + 1], scale_value(ea[i]));
#pragma unroll
          for (int j = 0; j < FN; ++j) acc[I0 + i][j] = mma<true>(wb[j], wa, acc[I0 + i][j]);
        }
      }
    }
  }

  template <class L, class RA, class RB>
  __device__ static __forceinline__ void straight(int n, int wave, uint16_t* lds, L load, RA read_a, RB read_b, Acc& acc) {
    constexpr int AHEAD = S::STAGES - 1, LOADS = A::PER + B::PER;      // loads of a slab, one more for scales
    static_assert(A::WORK == S::NT && B::WORK == S::NT, "of all wavefronts");
#pragma unroll
    for (int t = 0; t < AHEAD; ++t)
      if (t < n) load(t);
    for (int t = 0; t < n; ++t) {
      if (AHEAD == 1 || t + AHEAD > n) loads_done();
      else if (wave < SCALE_WAVES) loads_left<(LOADS + 1) * (AHEAD - 1)>();
      else loads_left<LOADS * (AHEAD - 1)>();
      group_barrier();      // slab t is there, and nobody reads slab t - 1 any more
      if (t + AHEAD < n) load(t + AHEAD);
      const uint16_t* const s = lds + t % S::STAGES * STAGE;
      v8i fa[FM], fb[FN];
      int ea[FM], eb[FN];
#pragma unroll
      for (int j = 0; j < FN; ++j) read_b(s, j, t, fb[j], eb[j]);
#pragma unroll
      for (int i = 0; i < FM; ++i) read_a(s, i, t, fa[i], ea[i]);
      multiply<0, FM>(fa, ea, fb, eb, acc);
    }
    lds_done();
    group_barrier();
  }
};

}  // namespace obl
