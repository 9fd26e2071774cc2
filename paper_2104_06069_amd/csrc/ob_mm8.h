// One workgroup's tile of C = A B^T with operands of 8 bits and a scale for each 128 columns of K, summed in binary32 on the
// matrix cores (gfx950), in one of two ways:
//   8-bit instructions, which take 128 columns at once and apply both operands' scales, powers of two, as they multiply: 4.7
//   PFLOP/s.  They cut each of eight adjacent products off 13 bits below the largest power of two among them before they sum them in
//   binary32, which makes 1.5e-5 (2-norm, normal numbers), whatever K is: far below the rounding of a 16-bit result.
//   WIDE, for binary32 results: operands made bfloat16 in registers, scales applied, both exactly for numbers from bfloat16's smallest, 2^-133,
//   to its largest, and the instructions for those, which lose nothing before binary32 (7e-8 at K = 8192): half the rate.
//
// An operand's rows are K bytes, K a multiple of 128 and zeros behind the matrix, so that a slab of 128 columns is always whole.  In
// LDS a row of it is eight pieces of 16 bytes, in an order permuted by the row's number so that lanes that read the same piece of
// their rows meet in no bank.  Lane (q, i) of a product gets pieces q and q + 4 of its row, for both operands alike.  Beside a slab lie the scales of
// its rows, four bytes each, for the four slabs of a group.
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

// Memory from p on, as the loads that go straight to LDS take it: an offset for each lane and one for all, 32 bits each
typedef __amdgpu_buffer_rsrc_t Buffer;
__device__ __forceinline__ Buffer buffer_of(const uint8_t* p, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), 0, (int)bytes, 0x00027000);
}

// BR rows of a slab, brought into LDS by NT threads
template <int BR, int NT>
struct Rows8 {
  static constexpr int PER = BR * 8 / NT, STEP = NT / 8;      // pieces a thread fetches, rows between them
  static_assert(PER * NT == BR * 8 && STEP % 8 == 0, "whole passes, of the same permutation");
  Buffer memory;
  int off[PER];

  __device__ void init(const Operand8& o, int r0, int tid) {
    memory = buffer_of(o.p + (int64_t)r0 * o.ld, min(o.rows - r0, BR) * o.ld);
    const int row = tid / 8, at = ((tid % 8) ^ (row & 7)) * 16;
#pragma unroll
    for (int j = 0; j < PER; ++j) off[j] = min(row + j * STEP, o.rows - 1 - r0) * (int)o.ld + at;      // (rows past the last repeat one that exists)
  }
  __device__ __forceinline__ void load(int slab, uint8_t* lds, int wave, int j) const {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(memory, in_lds<void>(lds + wave * 1024 + j * NT * 16), 16, off[j], slab * BLOCK8, 0, 0);
  }
};

// The scales of 64 rows, a lane each, for the group of four slabs that a slab is in
struct Scales8 {
  Buffer memory;
  int off;
  __device__ void init(const uint8_t* scales, int64_t ld, int rows, int shift, int first, int lane) {
    const int scale0 = first < rows ? first >> shift : 0, high = min(((rows - 1) >> shift) + 1 - scale0, 64);      // (rows of scales)
    memory = buffer_of(scales + scale0 * ld, high * ld);
    off = ((min(first + lane, rows - 1) >> shift) - scale0) * (int)ld;
  }
  __device__ __forceinline__ void load(int slab, uint8_t* lds) const {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(memory, in_lds<void>(lds), 4, off, slab / 4 * 4, 0, 0);
  }
};

// B's numbers are e4m3
template <int FORMAT>
__device__ __forceinline__ v4f mma8(v8i b, int scale_b, v8i a, int scale_a, v4f c) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, c, 0, FORMAT == E4M3 ? 0 : 1, 0, scale_b, 0, scale_a);
}

// Eight of a lane's bytes times the scale, as bfloat16: exact with scales from 2^-124 (e4m3) and 2^-117 (e5m2) on, by which the smallest numbers are
// bfloat16's
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
  static constexpr int BM = S::BM, BN = S::BN, FM = S::FM, FN = S::FN;
  static_assert(S::BK * 2 == BLOCK8, "slabs of a block");      // (BK of pairs of bytes)
  static constexpr int THREADS = S::WAVES * 64;                // of a team
  using A = Rows8<BM, THREADS>;
  using B = Rows8<BN, THREADS>;
  static constexpr int SCALE_WAVES = (BM + BN) / 64, SCALES = (BM + BN) * BLOCK8;      // (64 rows' scales a load); where a slab's scales begin
  static_assert(SCALE_WAVES <= S::WAVES, "a row's scales for each lane");
  static constexpr int STAGE = (BM + BN) * (BLOCK8 + 4);
  static constexpr int SUMS = Results<S>::LDS_BYTES, ENDS = SUMS + (S::TEAMS - 1) * S::WAVES * FM * FN * 1024;      // (the second team's, behind the results)
  static constexpr int LDS_BYTES = S::TEAMS * S::STAGES * STAGE > ENDS ? S::TEAMS * S::STAGES * STAGE : ENDS;
  typedef v4f Acc[FM][FN];

  // Slabs t0 .. t0 + n - 1 of K.  The layout of acc is Product's.  With two teams each has slabs of its own, every second one, and
  // the first one has the sums of both at the end.
  __device__ static void run(const Operand8& a, const Operand8& b, int r0, int c0, int t0, int n, uint8_t* lds, Acc& acc) {
    const int tid = threadIdx.x % THREADS, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int team = __builtin_amdgcn_readfirstlane((int)threadIdx.x / THREADS);
    uint8_t* const own = lds + team * S::STAGES * STAGE;
    const auto slab_at = [&](int t) { return t0 + t * S::TEAMS + team; };
    const int wm = wave / S::WN, wn = wave % S::WN;
    A sa;
    B sb;
    sa.init(a, r0, tid);
    sb.init(b, c0, tid);
    const bool of_a = wave < BM / 64;
    Scales8 scales;
    scales.init(of_a ? a.scales : b.scales, of_a ? a.ld_scales : b.ld_scales, of_a ? a.rows : b.rows, of_a ? a.shift : b.shift,
                of_a ? r0 + wave * 64 : c0 + wave * 64 - BM, lane);
    const auto load = [&](int t) {
      uint8_t* const s = own + t % S::STAGES * STAGE;
#pragma unroll
      for (int j = 0; j < A::PER; ++j) sa.load(slab_at(t), s, wave, j);
#pragma unroll
      for (int j = 0; j < B::PER; ++j) sb.load(slab_at(t), s + BM * BLOCK8, wave, j);
      if (wave < SCALE_WAVES) scales.load(slab_at(t), s + SCALES + wave * 256);
    };
    // Where a lane's pieces q and q + 4 of its row, and that row's scales, lie in a slab; fragments are 16 rows apart
    const int i = lane & 15, row_a = wm * (BM / S::WM) + i, row_b = BM + wn * (BN / S::WN) + i, piece = ((lane >> 4) ^ (i & 7)) * 16;
    const int a_lo = row_a * BLOCK8 + piece, a_hi = row_a * BLOCK8 + (piece ^ 64), b_lo = row_b * BLOCK8 + piece, b_hi = row_b * BLOCK8 + (piece ^ 64);
    const auto base = in_lds<uint8_t>(own);
    const auto read = [&](int lo, int hi, int row, int slab, int f, int t, v8i& to, int& e) {
      const int s = slab * STAGE;
      const v4i x = *(__attribute__((address_space(3))) const v4i*)(base + (s + lo) + f * 16 * BLOCK8);
      const v4i y = *(__attribute__((address_space(3))) const v4i*)(base + (s + hi) + f * 16 * BLOCK8);
      to = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
      e = *(base + (s + SCALES + row * 4 + (slab_at(t) & 3)) + f * 64);
    };
    const auto read_a = [&](int slab, int f, int t, v8i& to, int& e) { read(a_lo, a_hi, row_a, slab, f, t, to, e); };
    const auto read_b = [&](int slab, int f, int t, v8i& to, int& e) { read(b_lo, b_hi, row_b, slab, f, t, to, e); };
    if constexpr (S::TURNS) turns(n, load, read_a, read_b, acc);
    else straight((n + S::TEAMS - 1) / S::TEAMS, (n + S::TEAMS - 1 - team) / S::TEAMS, wave, load, read_a, read_b, acc);
    if constexpr (S::TEAMS > 1) {
      static_assert(S::TEAMS == 2, "one other team's sums");
      float* const at = reinterpret_cast<float*>(lds + SUMS) + (wave * FM * FN * 64 + lane) * 4;
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
          if (team) *in_lds<v4f>(at + (i * FN + j) * 256) = acc[i][j];
      lds_done();
      group_barrier();
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
          if (!team) acc[i][j] += *in_lds<const v4f>(at + (i * FN + j) * 256);
    }
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

  // n slabs, of `rounds` that every team waits through
  template <class L, class RA, class RB>
  __device__ static __forceinline__ void straight(int rounds, int n, int wave, L load, RA read_a, RB read_b, Acc& acc) {
    constexpr int AHEAD = S::STAGES - 1, LOADS = A::PER + B::PER;      // loads of a slab, one more for scales
#pragma unroll
    for (int t = 0; t < AHEAD; ++t)
      if (t < n) load(t);
    for (int t = 0; t < rounds; ++t) {
      if (AHEAD == 1 || t + AHEAD > n) loads_done();
      else if (wave < SCALE_WAVES) loads_left<(LOADS + 1) * (AHEAD - 1)>();
      else loads_left<LOADS * (AHEAD - 1)>();
      group_barrier();      // slab t is there, and nobody reads slab t - 1 any more
      if (S::TEAMS > 1 && t >= n) break;      // (the last round: the barrier below is next for everybody)
      if (t + AHEAD < n) load(t + AHEAD);
      const int s = t % S::STAGES;
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

  // Product's turns, two a slab: each with half of a wavefront's rows, the first with its columns' operands for both.
  template <class L, class RA, class RB>
  __device__ static __forceinline__ void turns(int n, L load, RA read_a, RB read_b, Acc& acc) {
    const bool second = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) >= S::WAVES / 2;
    constexpr int HALF = FM / 2;
    if (n > 0) {
      load(0);
      loads_done();
      group_barrier();
      if (second) {
        if (n > 1) load(1);
        group_barrier();
      }
      for (int t = 0; t < n; ++t) {
        const int s = t & 1;
        v8i fa[HALF], fb[FN];
        int ea[HALF], eb[FN];
#pragma unroll
        for (int j = 0; j < FN; ++j) read_b(s, j, t, fb[j], eb[j]);
#pragma unroll
        for (int i = 0; i < HALF; ++i) read_a(s, i, t, fa[i], ea[i]);
        if (!second && t + 1 < n) load(t + 1);
        lds_done();
        group_barrier();
        __builtin_amdgcn_s_setprio(1);
        multiply<0, HALF>(fa, ea, fb, eb, acc);
        // (here, and not behind the barrier beside the second half's: both halves' operands do not fit in registers)
#pragma unroll
        for (int i = 0; i < HALF; ++i)
#pragma unroll
          for (int j = 0; j < FN; ++j) asm volatile("" : "+v"(acc[i][j]));
        __builtin_amdgcn_s_setprio(0);
        group_barrier();
#pragma unroll
        for (int i = 0; i < HALF; ++i) read_a(s, HALF + i, t, fa[i], ea[i]);
        if (second) loads_done();
        else lds_done();
        group_barrier();
        if (second && t + 2 < n) load(t + 2);
        __builtin_amdgcn_s_setprio(1);
        multiply<HALF, HALF>(fa, ea, fb, eb, acc);
        __builtin_amdgcn_s_setprio(0);
        if (!second) loads_done();
        group_barrier();
      }
      if (!second) group_barrier();
    }
  }
};

// Many tiles of 256 x 256, results of adjacent eights, K of two slabs or more: workgroups that stay, one on a CU, and go from tile to
// tile without a pause in their loads.  A wavefront has a SIMD for itself and 128 x 128 of a tile.  It goes through its columns'
// fragments one after the other, with all of its rows': beside the products of one column it reads the next column's operand from LDS, and
// beside those of the last one, row by row as they are done with, the next slab's rows.  So A's part of a slab is done with when its
// columns begin, and the first half of B's when they are half through, and what is free is loaded again at once, for the slab after the
// next, which may be the next tile's: at Q, before column 3, A and the first columns; at P, before the last column, scales and the last
// columns.  Each is waited for a slab and a half after that, at the P or Q before it is read.  Loads are spread over the products: a
// wavefront that waits for its turn at the CU's loads issues no products (all of a slab's at once: 56 cycles a product in place of 44).
// Results go out while the next tile's products run: nothing waits for them but their own turn in the count of loads.
//   16-bit results   8192^3 in 417 us, 2.63 PFLOP/s (the library's product with one scale for each matrix: 2.62 to 2.71); 16384 x 8192 by 2048 226 us
//   binary32         a row's operand is made bfloat16 once a slab, a column's once a column: 8192 x 2048 by 32768 in 675 us, 1.63 PFLOP/s (the
//                    library's bfloat16 product at 8192^3: 1.31); with two rows' products in turn, which need more registers, 730
constexpr int ADD_F32 = 3;      // of types of results: binary32, added to what is there
template <int FORMAT, int OUT>
struct Flow8 {
  static constexpr bool WIDE = OUT == F32 || OUT == ADD_F32;
  static constexpr int BM = 256, BN = 256, NT = 256, FM = 8, FN = 8;
  using A = Rows8<BM, NT>;
  using B = Rows8<BN, NT>;
  static constexpr int SCALES = (BM + BN) * BLOCK8, STAGE = SCALES + (BM + BN) * 4;
  static constexpr int PITCH = 272, RESULTS = 16 * PITCH, LDS_BYTES = 2 * STAGE + 4 * RESULTS;      // (16 rows of 128 results a wavefront, four banks apart)
  static_assert(A::PER == 8 && B::PER == 8, "the loads below");
  static constexpr int STORES = WIDE ? FM * FN : FM * 4;      // of a tile, whatever part of it exists
  static constexpr int BEHIND = STORES < 45 ? STORES : 45;    // (a count of loads goes up to 63)

  struct Loads {      // of a tile, by a wavefront
    A a;
    B b;
    Scales8 sa, sb;
    __device__ void aim(const Operand8& oa, const Operand8& ob, int r0, int c0, int tid) {
      const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
      a.init(oa, r0, tid);
      b.init(ob, c0, tid);
      sa.init(oa.scales, oa.ld_scales, oa.rows, oa.shift, r0 + wave * 64, lane);
      sb.init(ob.scales, ob.ld_scales, ob.rows, ob.shift, c0 + wave * 64, lane);
    }
    // At Q: A, and columns 0 to 3 of both halves; at P: scales, and columns 4 to 7 of both
    __device__ __forceinline__ void at_q(int k, int slab, uint8_t* s, int wave) const {
      if (k < 8) a.load(slab, s, wave, k);
      else b.load(slab, s + BM * BLOCK8, wave, k < 10 ? k - 8 : k - 6);
    }
    __device__ __forceinline__ void at_p(int k, int slab, uint8_t* s, int wave) const {
      if (k == 0) sa.load(slab, s + SCALES + wave * 256);
      else if (k == 1) sb.load(slab, s + SCALES + (4 + wave) * 256);
      else b.load(slab, s + BM * BLOCK8, wave, k < 4 ? k : k + 2);
    }
  };

  // next(id) is the next tile's place, or none: {row, column}, row < 0
  template <class NEXT>
  __device__ static __forceinline__ void run(const Operand8& oa, const Operand8& ob, int n, void* out, int64_t ldo, uint8_t* lds, NEXT next) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / 2, wn = wave % 2, i16 = lane & 15, q = lane >> 4;
    int r0, c0, r1, c1;      // of the tile, and of the next one
    next(&r0, &c0);
    if (r0 < 0) return;
    Loads loads;
    loads.aim(oa, ob, r0, c0, tid);

    const int row_a = wm * 128 + i16, row_b = BM + wn * 128 + i16, piece = (q ^ (i16 & 7)) * 16;
    const int a_lo = row_a * BLOCK8 + piece, a_hi = row_a * BLOCK8 + (piece ^ 64), b_lo = row_b * BLOCK8 + piece, b_hi = row_b * BLOCK8 + (piece ^ 64);
    const auto base = in_lds<uint8_t>(lds);
    const auto read = [&](int lo, int hi, int row, int stage, int f, int slab, v8i& to, int& e) {
      const int s = stage * STAGE;
      const v4i x = *(__attribute__((address_space(3))) const v4i*)(base + (s + lo) + f * 16 * BLOCK8);
      const v4i y = *(__attribute__((address_space(3))) const v4i*)(base + (s + hi) + f * 16 * BLOCK8);
      to = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
      e = *(base + (s + SCALES + row * 4 + (slab & 3)) + f * 64);
    };
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int k = 0; k < 12; ++k) loads.at_q(k, t, lds + t * STAGE, wave);
#pragma unroll
      for (int k = 0; k < 6; ++k) loads.at_p(k, t, lds + t * STAGE, wave);
    }
    loads_done();
    group_barrier();
    // Operands: WIDE, made bfloat16 once for a slab (A) and for a column (B), from what was read two rows of products, or a column, before
    constexpr int RAW_A = WIDE ? 3 : FM;
    v8i fa[RAW_A], fb[2];
    int ea[RAW_A], eb[2];
    v8s wa[WIDE ? FM : 1][4], wb[WIDE ? 2 : 1][4];
    const auto widen_a = [&](int i) {
#pragma unroll
      for (int k = 0; k < 4; ++k) wa[WIDE ? i : 0][k] = widened<FORMAT>(fa[i % RAW_A][2 * k], fa[i % RAW_A][2 * k + 1], scale_value(ea[i % RAW_A]));
    };
    const auto widen_b = [&](int j, int k) { wb[WIDE ? j & 1 : 0][k] = widened<E4M3>(fb[j & 1][2 * k], fb[j & 1][2 * k + 1], scale_value(eb[j & 1])); };
    const auto multiply = [&](int i, int j, v4f& acc) {
      if constexpr (!WIDE) {
        acc = mma8<FORMAT>(fb[j & 1], eb[j & 1], fa[i], ea[i], acc);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) acc = mma<true>(wb[j & 1][k], wa[i][k], acc);
      }
    };
    read(b_lo, b_hi, row_b, 0, 0, 0, fb[0], eb[0]);
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      read(a_lo, a_hi, row_a, 0, i, 0, fa[i % RAW_A], ea[i % RAW_A]);
      if (WIDE && i < FM - 2) widen_a(i);
    }
    if constexpr (WIDE) {
#pragma unroll
      for (int k = 0; k < 4; ++k) widen_b(0, k);
    }
    int stage = 0;
    while (true) {
      v4f acc[FM][FN] = {};
      next(&r1, &c1);
      // AFTER: of a tile's first slab, behind the stores of the tile before (before the first tile everything has been waited for)
      const auto slab = [&](int t, auto after) {
        constexpr int MORE = decltype(after)::value ? BEHIND : 0;
        if (t + 2 == n && r1 >= 0) loads.aim(oa, ob, r1, c1, tid);
        const int one = t + 1 < n ? t + 1 : 0, two = t + 2 < n ? t + 2 : t + 2 - n;      // the slabs after this one, in their tile
        uint8_t* const here = lds + stage * STAGE;
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          const bool last = j == FN - 1;
          if (j == 3) {
            loads_left<18 + MORE>();      // (this slab's P: behind it the next slab's Q and P)
            group_barrier();
          }
          if (last) {
            loads_left<16 + MORE>();      // (the next slab's Q and scales: behind them its columns and the Q after that)
            group_barrier();
          }
          if (last) read(b_lo, b_hi, row_b, stage ^ 1, 0, one, fb[0], eb[0]);
          else read(b_lo, b_hi, row_b, stage, j + 1, t, fb[(j + 1) & 1], eb[(j + 1) & 1]);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int i = 0; i < FM; ++i) {
            if (WIDE && j == 0 && i < 2) widen_a(FM - 2 + i);
            multiply(i, j, acc[i][j]);
            if (WIDE && last && i >= 2) widen_a(i - 2);
            if (last) read(a_lo, a_hi, row_a, stage ^ 1, i, one, fa[i % RAW_A], ea[i % RAW_A]);
            if (WIDE && i >= 4) widen_b(j + 1, i - 4);
            if (j >= 3 && j < 7 && i % 3 == 0) loads.at_q((j - 3) * 3 + i / 3, two, here, wave);
            if (last && i < 6) loads.at_p(i, two, here, wave);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        stage ^= 1;
      };
      slab(0, std::true_type{});
#pragma unroll 1
      for (int t = 1; t < n; ++t) slab(t, std::false_type{});
      store(acc, oa.rows, ob.rows, out, ldo, r0, c0, lds + 2 * STAGE + wave * RESULTS, wm, wn, lane);
      if (r1 < 0) break;
      r0 = r1;
      c0 = c1;
    }
    loads_done();      // (what was loaded behind the last tile's end)
  }

 private:
  // A wavefront's results, sixteen rows at a time turned in LDS to 256 bytes of a row by sixteen lanes.  Always STORES stores: what lies outside
  // of the matrix has an offset outside of the buffer and is dropped.
  __device__ static __forceinline__ void store(const v4f (&acc)[FM][FN], int rows, int cols, void* out, int64_t ldo, int r0, int c0, uint8_t* own, int wm, int wn,
                                               int lane) {
    asm volatile("" : "+v"(lane));      // (offsets are made here, and not held through the products)
    const int high = min(rows - r0, BM), wide = min(cols - c0, BN);
    if constexpr (WIDE) {
      const Buffer to = buffer_of(static_cast<uint8_t*>(out) + (r0 * ldo + c0) * 4, ((high - 1) * ldo + wide) * 4);
      typedef unsigned v4u __attribute__((ext_vector_type(4)));
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        v4f old[FN];
        int at[FN];
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          const int r = wm * 128 + i * 16 + (lane & 15), c = wn * 128 + j * 16 + (lane >> 4) * 4;
          at[j] = r < high && c < wide ? (r * (int)ldo + c) * 4 : 0x7ffffff0;
          if constexpr (OUT == ADD_F32) old[j] = __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(to, at[j], 0, 0));
        }
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          v4f v = acc[i][j];
          asm volatile("" : "+a"(v)::"memory");
          if constexpr (OUT == ADD_F32) v += old[j];
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, v), to, at[j], 0, 0);
        }
      }
      return;
    }
    const Buffer to = buffer_of(static_cast<uint8_t*>(out) + (r0 * ldo + c0) * 2, ((high - 1) * ldo + wide) * 2);
    const auto mine = in_lds<uint8_t>(own);
#pragma unroll
    for (int i = 0; i < FM; ++i) {
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        v4f v = acc[i][j];
        asm volatile("" : "+a"(v)::"memory");      // (from where the products left it, and not before its turn: there are registers for sixteen rows)
        v4h h;
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = to_bits(v[e], OUT == BF16);
        *(__attribute__((address_space(3))) v2i*)(mine + (lane & 15) * PITCH + j * 32 + (lane >> 4) * 8) = __builtin_bit_cast(v2i, h);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int row = u * 4 + (lane >> 4), piece = lane & 15, r = wm * 128 + i * 16 + row, c = wn * 128 + piece * 8;
        const v4i v = *(__attribute__((address_space(3))) const v4i*)(mine + row * PITCH + piece * 16);
        const int at = r < high && c < wide ? (r * (int)ldo + c) * 2 : 0x7ffffff0;
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(unsigned __attribute__((ext_vector_type(4))), v), to, at, 0, 0);
      }
    }
  }
};

}  // namespace obl
