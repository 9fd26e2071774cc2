// Core of the matrix operators (gfx950): one workgroup's tile of C = A B^T with 16-bit operands and binary32
// accumulation, on the matrix cores.  Included by ob_matrix.hip only.
//
// An operand is a matrix of `rows` rows (the tile's M or N side) and K columns, in one of two orders: KC, element (r, k)
// at p[r * ld + k], or KS, element (r, k) at p[k * ld + r].  It has one or two terms (planes `term` elements apart): with
// two, its value is their sum, a binary16 number and the binary16 rounding of what that left over (22 bits).  The product
// of two two-term operands leaves out the product of the second terms, 2^-22 of the result.
//
// What bounds such a tile is the rate of the matrix instructions, and next to it LDS: a wavefront of a 256 x 256 tile owns
// 128 x 64 of it and reads 12 KB of LDS for each 32 columns of K, 768 of the 1024 cycles that the eight wavefronts' matrix
// instructions take.  The wavefronts are therefore two groups that take turns, half a step apart: while one reads its
// operands from LDS (and starts the loads of the next K slab from memory straight into LDS), the other has the matrix
// cores.  Measured at 8192^3: 1190 to 1310 TFLOP/s with bfloat16 operands (the library's product of the same: 1314), with
// two terms 1370 to 1495 TFLOP/s of matrix instructions (three products out of each two slabs read); 128 x 128 tiles of four
// wavefronts 1130 and 1090, 64 x 64 ones 760.
//
// LDS holds 16-byte pieces in the order in which the loads bring them.  Which piece of its row a lane fetches is permuted
// by the row's number, so that the reads below do not meet in the same banks.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace obm {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef short v8s_any __attribute__((ext_vector_type(8), aligned(2)));   // at any 2-byte address
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));
typedef unsigned long long v2u __attribute__((ext_vector_type(2)));

enum { KC = 0, KS = 1 };

template <class T>
__device__ __forceinline__ __attribute__((address_space(3))) T* in_lds(const void* p) {
  return (__attribute__((address_space(3))) T*)p;
}

template <bool BF>
__device__ __forceinline__ v4f mma(v8s a, v8s b, v4f c) {
  if constexpr (BF) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b, a), __builtin_bit_cast(v8b, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
}

struct Operand {
  const uint16_t* p;
  int64_t term;    // elements from the first term's plane to the second's
  int64_t ld;
  int rows;        // >= 1
  bool direct;     // every 16-byte piece lies at a 16-byte address (and rows % 8 == 0 in the KS order)
};

// BR rows by BK columns of an operand, brought into LDS by NT threads
template <int FORM, int BR, int BK, int NT>
struct Slab {
  static constexpr int PIECES = FORM == KC ? BK / 8 : BR / 8;      // of 8 elements, in one row of LDS
  static constexpr int ALL = BR * BK / 8, WORK = ALL < NT ? ALL : NT;   // threads that fetch: whole wavefronts
  static constexpr int PER = ALL / WORK, STEP = WORK / PIECES;     // pieces each of them fetches, LDS rows between those
  static_assert(BK == 32 || BK == 64, "the permutations below");
  static_assert(PER * WORK == ALL && WORK % 64 == 0 && WORK % PIECES == 0 && (PER == 1 || STEP % 8 == 0), "whole passes; every one, or every second one, of the same permutation");

  __device__ static int turn(int row) {
    if constexpr (FORM == KC) return BK == 64 ? row & 7 : (row >> 1) & 3;
    else return (((row & 3) | ((row >> 1) & 4)) << 1) & (PIECES - 1);
  }

  static constexpr int OFFS = FORM == KC ? PER : PER > 1 && STEP % 16 ? 2 : 1;
  int off[OFFS];     // elements from the tile's first

  __device__ void init(const Operand& o, int r0, int tid) {
    const int row = tid / PIECES, at = ((tid % PIECES) ^ turn(row)) * 8;
    if constexpr (FORM == KC) {
#pragma unroll
      for (int j = 0; j < PER; ++j) off[j] = (int)((min(r0 + row + j * STEP, o.rows - 1) - r0) * o.ld) + at;
    } else {
#pragma unroll
      for (int j = 0; j < OFFS; ++j) off[j] = (int)(row * o.ld) + min(r0 + (tid % PIECES ^ turn(row + j * STEP)) * 8, o.rows - 8) - r0;
    }
  }

  // A slab whose BK columns all exist, of an operand with `direct`: rows past the last repeat one that exists.
  // ONCE: what is read by this workgroup alone (not kept in the caches).
  template <bool ONCE = false>
  __device__ void load(const Operand& o, int term, int r0, int k0, uint16_t* lds, int wave) const {
    if (WORK < NT && wave >= WORK / 64) return;
    const uint16_t* const base = o.p + term * o.term;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const uint16_t* src;
      if constexpr (FORM == KC) src = base + (int64_t)r0 * o.ld + k0 + off[j];
      else src = base + (int64_t)(k0 + j * STEP) * o.ld + r0 + off[j % OFFS];
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src, in_lds<void>(lds + wave * 512 + j * WORK * 8), 16, 0, ONCE ? 2 : 0);
    }
  }

  // Through registers, from any address: fetch() starts a slab's loads, put() takes them to LDS.  Where all of the slab
  // exists (KC: rows past the last repeat one that does), with the offsets of load():
  typedef v8s Fetched[PER];
  __device__ static bool exists(const Operand& o, int r0, int k0, int K) { return k0 + BK <= K && (FORM == KC || r0 + BR <= o.rows); }
  __device__ void fetch_whole(const Operand& o, int r0, int k0, int tid, Fetched& v) const {
    if (WORK < NT && tid >= WORK) return;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const uint16_t* src;
      if constexpr (FORM == KC) src = o.p + (int64_t)r0 * o.ld + k0 + off[j];
      else src = o.p + (int64_t)(k0 + j * STEP) * o.ld + r0 + off[j % OFFS];
      v[j] = *reinterpret_cast<const v8s_any*>(src);
    }
  }
  __device__ static void put_whole(const Fetched& v, uint16_t* lds, int tid) {
    if (WORK < NT && tid >= WORK) return;
#pragma unroll
    for (int j = 0; j < PER; ++j) *in_lds<v8s>(lds + (j * WORK + tid) * 8) = v[j];
  }
  // Any slab.  Columns from K on are zeros.
  // How many of the eight elements of piece j exist (8: all; 0 or less: none), and the width of a row in memory
  __device__ static int piece_left(const Operand& o, int r0, int k0, int K, int tid, int j, int* r, int* c) {
    const int row = tid / PIECES + j * STEP, at = (tid % PIECES ^ turn(row)) * 8;
    *r = FORM == KC ? min(r0 + row, o.rows - 1) : k0 + row;
    *c = FORM == KC ? k0 + at : r0 + at;
    return *r < (FORM == KC ? o.rows : K) ? (FORM == KC ? K : o.rows) - *c : 0;
  }
  __device__ static void fetch(const Operand& o, int r0, int k0, int K, int tid, Fetched& v) {
    if (WORK < NT && tid >= WORK) return;
    const int width = FORM == KC ? K : o.rows;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      int r, c;
      const int left = piece_left(o, r0, k0, K, tid, j, &r, &c);
      const uint16_t* const src = o.p + (int64_t)r * o.ld + c;
      v[j] = v8s{};
      if (left > 0 && width >= 8) {
        v[j] = *reinterpret_cast<const v8s_any*>(src + min(left - 8, 0));      // at the end of a row: its last eight
      } else if (left > 0) {
#pragma unroll
        for (int e = 0; e < 7; ++e)
          if (e < left) v[j][e] = (short)src[e];
      }
    }
  }
  __device__ static void put(const Operand& o, int r0, int k0, int K, int tid, const Fetched& v, uint16_t* lds) {
    if (WORK < NT && tid >= WORK) return;
    const int width = FORM == KC ? K : o.rows;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      int r, c;
      const int left = piece_left(o, r0, k0, K, tid, j, &r, &c);
      v8s piece = v[j];
      if (left > 0 && left < 8 && width >= 8) {      // moved down to where they belong, zeros behind them
        const v2u w = __builtin_bit_cast(v2u, piece);
        const int s = (8 - left) * 16;
        v2u z;
        z.x = s >= 64 ? w.y >> (s - 64) : (w.x >> s) | (w.y << (64 - s));
        z.y = s >= 64 ? 0 : w.y >> s;
        piece = __builtin_bit_cast(v8s, z);
      }
      *in_lds<v8s>(lds + (j * WORK + tid) * 8) = piece;
    }
  }
  __device__ static void load_any(const Operand& o, int r0, int k0, int K, uint16_t* lds, int tid) {
    Fetched v;
    fetch(o, r0, k0, K, tid, v);
    put(o, r0, k0, K, tid, v, lds);
  }

  // Operand registers of a 16x16x32 product: lane (q, i) gets row f0 + i, columns 32 kk + 8 q + 0..7 of the slab.
  __device__ static v8s fragment(const uint16_t* lds, int f0, int kk, int lane) {
    const int i = lane & 15, q = lane >> 4;
    if constexpr (FORM == KC) {
      return *in_lds<const v8s>(lds + (f0 + i) * BK + (((kk * 4 + q) ^ turn(i)) * 8));
    } else {
      // sixteen lanes read 4 columns by 16 rows, and get them transposed
      const int k = kk * 32 + 8 * q + (i >> 2), piece = (f0 >> 3) + ((i & 3) >> 1);
      const uint16_t* const a = lds + k * BR + ((piece ^ turn(k)) * 8) + (i & 1) * 4;     // (turn(k) == turn(k + 4))
      const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(in_lds<v4s>(a));
      const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(in_lds<v4s>(a + 4 * BR));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
  }
};

__device__ __forceinline__ void group_barrier() {
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
}
__device__ __forceinline__ void loads_done() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void lds_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Until at most n of this wavefront's loads are under way
template <int n>
__device__ __forceinline__ void loads_left() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(n) : "memory");
}

// WM x WN wavefronts share out a tile.  STAGES: slabs in LDS at once.  Eight (two on each SIMD) take turns as described above,
// with two slabs; fewer do not wait for each other in between: the loads of STAGES - 1 slabs are under way, and what one workgroup
// leaves idle another one on the CU uses.  With two TEAMS the tile has twice as many wavefronts, and each team half the columns of
// each slab: for tiles that have a CU to themselves, where every read of LDS is waited for.
template <int BM_, int BN_, int BK_, int WM_, int WN_, int STAGES_ = 2, int TEAMS_ = 1>
struct Shape {
  static constexpr int BM = BM_, BN = BN_, BK = BK_, WM = WM_, WN = WN_, STAGES = STAGES_, TEAMS = TEAMS_;
  static constexpr int WAVES = WM * WN, NT = WAVES * TEAMS * 64;
  static constexpr bool TURNS = WAVES == 8;
  static_assert(TEAMS == 1 || (!TURNS && BK / 32 % TEAMS == 0), "whole steps of 32 columns for each team");
  static_assert(!TURNS || STAGES == 2, "two slabs");
  static constexpr int FM = BM / WM / 16, FN = BN / WN / 16;
};

// The tile's results, turned in LDS from the matrix cores' layout to rows.  Each wavefront has a part of LDS of its own and
// turns up to four times sixteen of its rows at a time.
template <class S>
struct Results {
  static constexpr int WIDTH = S::BN / S::WN, GROUP = S::FM < 4 ? S::FM : 4, ROWS = GROUP * 16;
  static constexpr int STRIDE = WIDTH + 4;        // floats: rows four banks apart
  static constexpr int LDS_BYTES = S::WAVES * ROWS * STRIDE * 4;

  // For four adjacent columns of a row at a time (ROWWISE), or four adjacent rows of a column: calls before(row, column), for
  // what has to be read beside them, and then after(row, column, values, what before() gave).
  template <bool ROWWISE, class F, class G>
  __device__ static __forceinline__ void pass(const float* own, int r0, int c0, F before, G after) {
    constexpr int EACH = ROWS * WIDTH / 256, BATCH = EACH < 4 ? EACH : 4;      // pieces a lane; how many are under way at once
    const int lane = threadIdx.x & 63;
#pragma unroll 1
    for (int k0 = lane; k0 < EACH * 64; k0 += BATCH * 64) {
      v4f v[BATCH], w[BATCH];
#pragma unroll
      for (int u = 0; u < BATCH; ++u) {
        const int k = k0 + u * 64;
        if constexpr (ROWWISE) {
          const int r = k / (WIDTH / 4), c = k % (WIDTH / 4) * 4;
          v[u] = *in_lds<const v4f>(own + r * STRIDE + c);
          w[u] = before(r0 + r, c0 + c);
        } else {
          const int c = k / (ROWS / 4), r = k % (ROWS / 4) * 4;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[u][e] = *in_lds<const float>(own + (r + e) * STRIDE + c);
          w[u] = before(r0 + r, c0 + c);
        }
      }
#pragma unroll
      for (int u = 0; u < BATCH; ++u) {
        const int k = k0 + u * 64;
        if constexpr (ROWWISE) after(r0 + k / (WIDTH / 4), c0 + k % (WIDTH / 4) * 4, v[u], w[u]);
        else after(r0 + k % (ROWS / 4) * 4, c0 + k / (ROWS / 4), v[u], w[u]);
      }
    }
  }

  // The same for eight adjacent elements at a time; values and before()'s are pairs of v4f.
  struct Eight {
    v4f a, b;
  };
  template <bool ROWWISE, class F, class G>
  __device__ static __forceinline__ void pass8(const float* own, int r0, int c0, F before, G after) {
    constexpr int EACH = ROWS * WIDTH / 512, BATCH = EACH < 2 ? EACH : 2;
    static_assert(EACH >= 1, "a piece for every lane");
    const int lane = threadIdx.x & 63;
#pragma unroll 1
    for (int k0 = lane; k0 < EACH * 64; k0 += BATCH * 64) {
      Eight v[BATCH], w[BATCH];
#pragma unroll
      for (int u = 0; u < BATCH; ++u) {
        const int k = k0 + u * 64;
        if constexpr (ROWWISE) {
          const int r = k / (WIDTH / 8), c = k % (WIDTH / 8) * 8;
          v[u].a = *in_lds<const v4f>(own + r * STRIDE + c);
          v[u].b = *in_lds<const v4f>(own + r * STRIDE + c + 4);
          w[u] = before(r0 + r, c0 + c);
        } else {
          const int c = k / (ROWS / 8), r = k % (ROWS / 8) * 8;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            v[u].a[e] = *in_lds<const float>(own + (r + e) * STRIDE + c);
            v[u].b[e] = *in_lds<const float>(own + (r + e + 4) * STRIDE + c);
          }
          w[u] = before(r0 + r, c0 + c);
        }
      }
#pragma unroll
      for (int u = 0; u < BATCH; ++u) {
        const int k = k0 + u * 64;
        if constexpr (ROWWISE) after(r0 + k / (WIDTH / 8), c0 + k % (WIDTH / 8) * 8, v[u], w[u]);
        else after(r0 + k % (ROWS / 8) * 8, c0 + k / (ROWS / 8), v[u], w[u]);
      }
    }
  }

  // by(own, r0, c0): what to do with `own`, the rows r0 .. and columns c0 .. of the tile that this wavefront has turned (see
  // pass()).  To be called after Product::run, whose last barrier ends the reads of LDS.
  template <class F>
  __device__ static __forceinline__ void visit(const v4f (&acc)[S::FM][S::FN], uint16_t* lds, F by) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (S::TEAMS > 1 && wave >= S::WAVES) return;      // (the first team has the sums)
    const int r0 = wave / S::WN * (S::BM / S::WM), c0 = wave % S::WN * WIDTH;
    float* const own = reinterpret_cast<float*>(lds) + wave * ROWS * STRIDE;
#pragma unroll
    for (int g = 0; g < S::FM / GROUP; ++g) {
#pragma unroll
      for (int i = 0; i < GROUP; ++i)
#pragma unroll
        for (int j = 0; j < S::FN; ++j)
          *in_lds<v4f>(own + (i * 16 + (lane & 15)) * STRIDE + j * 16 + 4 * (lane >> 4)) = acc[g * GROUP + i][j];
      lds_done();
      by(own, r0 + g * ROWS, c0);
      lds_done();
    }
  }
  // after(row, column, values of four adjacent columns) for all of the tile
  template <class G>
  __device__ static __forceinline__ void by_rows(const v4f (&acc)[S::FM][S::FN], uint16_t* lds, G after) {
    visit(acc, lds, [&](const float* own, int r0, int c0) {
      pass<true>(own, r0, c0, [](int, int) { return v4f{}; }, [&](int r, int c, v4f v, v4f) { after(r, c, v); });
    });
  }
};

// What the operands may be.  WHOLE: `direct`, K a multiple of BK; TAIL: `direct`, any K, the last slab through registers once
// the others are done; ANY: every slab through registers, the next one's loads under way while one is multiplied (there are
// not enough registers for that beside a 256 x 256 tile's).
enum { WHOLE = 0, TAIL = 1, ANY = 2 };

template <class S, bool BF, int FA, int FB, int TA, int TB, int MODE>
struct Product {
  static constexpr int BM = S::BM, BN = S::BN, BK = S::BK, FM = S::FM, FN = S::FN;
  static_assert(MODE == WHOLE || (TA == 1 && TB == 1), "load_any has one term");
  using A = Slab<FA, BM, BK, S::NT>;
  using B = Slab<FB, BN, BK, S::NT>;
  static constexpr int STAGE = (TA * BM + TB * BN) * BK;
  static constexpr int LDS_BYTES = S::STAGES * STAGE * 2 > Results<S>::LDS_BYTES ? S::STAGES * STAGE * 2 : Results<S>::LDS_BYTES;
  typedef v4f Acc[FM][FN];

  // Lane (q, i) of wavefront (wm, wn): acc[x][y][e] is row wm * BM / WM + 16 x + i, column wn * BN / WN + 16 y + 4 q + e.
  // K columns from k0 on; K >= 1.
  __device__ static void run(const Operand& a, const Operand& b, int r0, int c0, int k0, int K, uint16_t* lds, Acc& acc) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int team = wave / S::WAVES, wm = wave % S::WAVES / S::WN, wn = wave % S::WN;
    A sa;
    B sb;
    sa.init(a, r0, tid);
    sb.init(b, c0, tid);
    const int n = MODE == ANY ? (K + BK - 1) / BK : K / BK, end = k0 + K;
    auto load = [&](int t) {
      uint16_t* const s = lds + t % S::STAGES * STAGE;
#pragma unroll
      for (int x = 0; x < TA; ++x) sa.load(a, x, r0, k0 + t * BK, s + x * BM * BK, wave);
#pragma unroll
      for (int y = 0; y < TB; ++y) sb.load(b, y, c0, k0 + t * BK, s + (TA * BM + y * BN) * BK, wave);
    };
    auto read = [&](const uint16_t* s, int kk, v8s (&fa)[TA][FM], v8s (&fb)[TB][FN]) {
#pragma unroll
      for (int y = 0; y < TB; ++y)
#pragma unroll
        for (int f = 0; f < FN; ++f) fb[y][f] = B::fragment(s + (TA * BM + y * BN) * BK, wn * (BN / S::WN) + f * 16, kk, lane);
#pragma unroll
      for (int x = 0; x < TA; ++x)
#pragma unroll
        for (int f = 0; f < FM; ++f) fa[x][f] = A::fragment(s + x * BM * BK, wm * (BM / S::WM) + f * 16, kk, lane);
    };
    // The matrix cores cut an addend's bits off below the sum's last few; where there are registers for it the small products
    // of second terms have sums of their own (for four 512 x 512 matrices 1.2e-6 in place of 2e-6 off).
    constexpr bool APART = TA == 2 && TB == 2 && !S::TURNS;
    v4f small[APART ? FM : 1][APART ? FN : 1] = {};
    auto multiply = [&](const v8s (&fa)[TA][FM], const v8s (&fb)[TB][FN]) {
#pragma unroll
      for (int x = 0; x < TA; ++x)
#pragma unroll
        for (int y = 0; y < TB; ++y)
          if (x + y < 2) {
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
              for (int j = 0; j < FN; ++j) {
                v4f& sum = APART && x + y ? small[i % (APART ? FM : 1)][j % (APART ? FN : 1)] : acc[i][j];
                sum = mma<BF>(fb[y][j], fa[x][i], sum);
              }
          }
    };
    if constexpr (MODE == ANY) through_registers(sa, sb, a, b, r0, c0, k0, end, n, team, lds, read, multiply);
    else if constexpr (S::TURNS) turns(n, lds, acc, load, read, multiply);
    else straight(n, wave, team, lds, load, read, multiply);
    if constexpr (APART) {
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] += small[i][j];
    }
    if (MODE == TAIL && n * BK < K) {
      A::load_any(a, r0, k0 + n * BK, end, lds, tid);
      B::load_any(b, c0, k0 + n * BK, end, lds + TA * BM * BK, tid);
      lds_done();
      group_barrier();
      steps(lds, team, read, multiply);
      lds_done();
      group_barrier();
    }
    if constexpr (S::TEAMS > 1) {      // the second team's sums to the first
      static_assert(S::TEAMS == 2 && S::WAVES * FM * FN * 1024 <= LDS_BYTES, "room for them");
      float* const at = reinterpret_cast<float*>(lds) + (wave % S::WAVES) * FM * FN * 256 + lane * 4;
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
      lds_done();
      group_barrier();
    }
  }

 private:
  // A team's share of a slab
  template <class R, class M>
  __device__ static __forceinline__ void steps(const uint16_t* s, int team, R read, M multiply) {
#pragma unroll
    for (int k = 0; k < BK / 32 / S::TEAMS; ++k) {
      v8s fa[TA][FM], fb[TB][FN];
      read(s, k * S::TEAMS + team, fa, fb);
      multiply(fa, fb);
    }
  }

  template <class L, class R, class M>
  __device__ static __forceinline__ void straight(int n, int wave, int team, uint16_t* lds, L load, R read, M multiply) {
    constexpr int AHEAD = S::STAGES - 1;
    constexpr int NA = TA * A::PER, NB = TB * B::PER;      // loads of a slab, of the wavefronts that have such
    const bool la = wave < A::WORK / 64, lb = wave < B::WORK / 64;
#pragma unroll
    for (int t = 0; t < AHEAD; ++t)
      if (t < n) load(t);
    for (int t = 0; t < n; ++t) {
      if (AHEAD == 1 || t + AHEAD > n) loads_done();
      else if (la && lb) loads_left<(NA + NB) * (AHEAD - 1)>();
      else if (lb) loads_left<NB * (AHEAD - 1)>();
      else if (la) loads_left<NA * (AHEAD - 1)>();
      else lds_done();
      group_barrier();      // slab t is there, and nobody reads slab t - 1 any more
      if (t + AHEAD < n) load(t + AHEAD);
      steps(lds + t % S::STAGES * STAGE, team, read, multiply);
    }
    lds_done();
    group_barrier();
  }

  template <class R, class M>
  __device__ static __forceinline__ void through_registers(const A& sa, const B& sb, const Operand& a, const Operand& b, int r0, int c0, int k0, int end, int n, int team, uint16_t* lds,
                                                           R read, M multiply) {
    const int tid = threadIdx.x;
    typename A::Fetched va;
    typename B::Fetched vb;
    const auto fetch = [&](int k) {
      if (A::exists(a, r0, k, end)) sa.fetch_whole(a, r0, k, tid, va);
      else A::fetch(a, r0, k, end, tid, va);
      if (B::exists(b, c0, k, end)) sb.fetch_whole(b, c0, k, tid, vb);
      else B::fetch(b, c0, k, end, tid, vb);
    };
    fetch(k0);
    for (int t = 0; t < n; ++t) {
      uint16_t* const s = lds + t % 2 * STAGE;      // nobody reads slab t - 2 after the barrier of t - 1
      const int k = k0 + t * BK;
      if (A::exists(a, r0, k, end)) A::put_whole(va, s, tid);
      else A::put(a, r0, k, end, tid, va, s);
      if (B::exists(b, c0, k, end)) B::put_whole(vb, s + TA * BM * BK, tid);
      else B::put(b, c0, k, end, tid, vb, s + TA * BM * BK);
      lds_done();
      group_barrier();
      if (t + 1 < n) fetch(k + BK);
      steps(s, team, read, multiply);
    }
    lds_done();
    group_barrier();
  }

  template <class L, class R, class M>
  __device__ static __forceinline__ void turns(int n, uint16_t* lds, Acc& acc, L load, R read, M multiply) {
    const bool second = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) >= S::WAVES / 2;
    // Turns are separated by barriers; the second group is one turn behind.  Slab t + 1 goes where slab t - 1 was: both
    // groups start it in the turn after the second group's last read of slab t - 1, and wait for it at the end of the turn
    // before the first group's first read.
    if (n > 0) {
      load(0);
      loads_done();
      group_barrier();
      if (second) {
        if (n > 1) load(1);
        group_barrier();
      }
      for (int t = 0; t < n; ++t) {
        const uint16_t* const s = lds + (t & 1) * STAGE;
#pragma unroll
        for (int kk = 0; kk < BK / 32; ++kk) {
          const bool last = kk == BK / 32 - 1;
          v8s fa[TA][FM], fb[TB][FN];
          read(s, kk, fa, fb);
          if (kk == 0 && !second && t + 1 < n) load(t + 1);
          if (last && second) loads_done();
          else lds_done();
          group_barrier();
          if (last && second && t + 2 < n) load(t + 2);
          __builtin_amdgcn_s_setprio(1);
          multiply(fa, fb);
          __builtin_amdgcn_s_setprio(0);
          if (last && !second) loads_done();
          group_barrier();
        }
      }
      if (!second) group_barrier();
    }
  }
};

// Workgroups are dealt to the eight dies in turn, each with a cache of its own: consecutive tiles go to one die.  -1: none.
__device__ __forceinline__ int tile_of_workgroup(int id, int tiles) {
  const int per = (tiles + 7) / 8, at = id >> 3, t = (id & 7) * per + at;
  return at < per && t < tiles ? t : -1;
}

// Tile t of nm x nn: bands of up to 4 rows of tiles, down a band's columns first, so that the tiles that run at the same
// time share operands.
__device__ __forceinline__ void tile_in_bands(int t, int nm, int nn, int* tm, int* tn) {
  const int band = t / (4 * nn), first = band * 4, height = min(4, nm - first), u = t - first * nn;
  *tm = first + u % height;
  *tn = u / height;
}

}  // namespace obm
