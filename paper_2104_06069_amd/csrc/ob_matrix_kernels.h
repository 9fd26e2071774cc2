// Kernels of the matrix operators (include/ob_matrix.h), on the tiles of ob_mm.h.  Included by ob_matrix.hip only.
//
// Times stated beside the kernels are calls among others of their kind, timed by events; those of single kernels of the
// orthogonalised update, marked P, are medians under the profiler, where they come out up to 17% longer (the two large gradients of
// an expert layer 2.54 ms there, 2.26 ms without).
#pragma once

#include <type_traits>

#include "ob_matrix_plan.h"
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

// Where tile t of `side` of a range of `size` starts.  With operands that go through registers the last tile is moved back to
// end where the range does, so that its slabs exist as a whole; what it shares with the one before is computed twice, and stored by
// that one.
template <int MODE>
__device__ __forceinline__ int tile_start(int t, int side, int size) {
  return MODE == ANY ? min(t * side, max(size - side, 0)) : t * side;
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

extern __shared__ __align__(1024) uint16_t lds_of_launch[];

// ---- expert layers -------------------------------------------------------------------------------------------------
struct Groups {
  const int32_t* offsets;
  int n, rows;
  // rows of group g, inside 0..rows whatever the table holds
  __device__ __forceinline__ void range(int g, int* lo, int* hi) const {
    *lo = min(max(offsets[g], 0), rows);
    *hi = max(min(offsets[g + 1], rows), *lo);
  }
};

// The groups' tiles of BM rows, one after the other, as every wavefront counts them, 64 groups at a time.  The host knows an
// upper bound of their number alone.
struct RowTile {
  int g, lo, rows, tm, tn;      // a tile's group, that group's first row and number of rows, and the tile's place among its tiles
};
template <int BM>
struct RowTiles {
  int lo, hi, own, upto;             // of group `lane` (of the first 64): rows, tiles, and tiles up to and with it
  int64_t total;                     // tiles of all groups (ranges that overlap can make it any number)
  __device__ __forceinline__ void look(const Groups& gr, int g0) {
    const int lane = threadIdx.x & 63;
    lo = hi = 0;
    if (g0 + lane < gr.n) gr.range(g0 + lane, &lo, &hi);
    upto = own = (hi - lo + BM - 1) / BM;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(upto, d);
      if (lane >= d) upto += o;
    }
  }
  __device__ __forceinline__ explicit RowTiles(const Groups& gr) {
    total = 0;
    for (int g0 = (gr.n - 1) / 64 * 64; g0 >= 0; g0 -= 64) {      // (the first 64 last: they stay)
      look(gr, g0);
      total += __builtin_amdgcn_readlane(upto, 63);
    }
  }
  // Tile `tile` of them and of the `width` columns of tiles; to be called once
  __device__ __forceinline__ RowTile find(const Groups& gr, int width, int tile) {
    RowTile out = {};
    int64_t before = 0;
    for (int g0 = 0; g0 < gr.n; g0 += 64) {
      if (g0) look(gr, g0);
      const unsigned long long past = __ballot((before + upto) * width > tile);
      if (past) {
        const int l = __builtin_amdgcn_readfirstlane(__ffsll((long long)past) - 1);
        const int tiles = __builtin_amdgcn_readlane(own, l);
        const int64_t first = before + __builtin_amdgcn_readlane(upto, l) - tiles;
        tile_in_bands((int)(tile - first * width), tiles, width, &out.tm, &out.tn);
        out.g = g0 + l;
        out.lo = __builtin_amdgcn_readlane(lo, l);
        out.rows = __builtin_amdgcn_readlane(hi, l) - out.lo;
        return out;
      }
      before += __builtin_amdgcn_readlane(upto, 63);
    }
    return out;
  }
};

// forward (x, W, y) and input_grad (dy, W transposed, dx): out[r] = a[r] W_g, a [rows, depth], out [rows, width].  FB: order
// of W as an operand of `width` rows.  Tiles of 256 are bounded by the matrix instructions, and by their results, which all CUs
// write at about the same time: 32768 rows over 16 groups, 8192 deep, 2048 wide in 1.07 ms, 1025 TFLOP/s; 16384 over 8, 1024 deep,
// 4096 wide in 176 us, 780.  Tiles of 64 are for calls with too few of those, which the latency of their slabs bounds: 4096 rows
// over 16 groups, 2048 deep, 512 wide in 28 us, 305 TFLOP/s.
struct RowsArgs {
  Groups groups;
  const uint16_t* a;
  const uint16_t* w;
  void* out;
  int64_t lda, ldw, ldo, w_stride;
  int depth, width, out_dtype;
  bool a_direct, w_direct;
};
template <class S, bool BF, int FB, int MODE>
__device__ __forceinline__ void rows_tile(const RowsArgs& p, const RowTile& t, int r0, int c0) {
  using P = Product<S, BF, KC, FB, 1, 1, MODE>;
  if (r0 >= t.rows || c0 >= p.width) return;
  const int col0 = c0;
  if constexpr (FB == KS) c0 = tile_start<MODE>(c0 / S::BN, S::BN, p.width);
  typename P::Acc acc = {};
  const Operand a{p.a + t.lo * p.lda, 0, p.lda, t.rows, p.a_direct};
  const Operand b{p.w + t.g * p.w_stride, 0, p.ldw, p.width, p.w_direct};
  P::run(a, b, r0, c0, 0, p.depth, lds_of_launch, acc);
  void* const out = static_cast<char*>(p.out) + t.lo * p.ldo * (p.out_dtype == F32 ? 4 : 2);
  store_tile<S, BF>(acc, lds_of_launch, out, p.out_dtype, p.ldo, r0, c0, t.rows, p.width, 0, col0);
}
template <class S, bool BF, int FB, int MODE>
__global__ __launch_bounds__(S::NT, 2) void k_experts_rows(RowsArgs p) {
  const int width = (p.width + S::BN - 1) / S::BN;
  RowTiles<S::BM> all(p.groups);
  const int tiles = (int)min(all.total * width, (int64_t)0x7fffff00);
  // A CU has one workgroup of 256 x 256 at a time.  Of the last round, if it would leave half the card or more idle, each tile is
  // split between two workgroups, or four.  (1088 tiles, 4.25 rounds, of K = 1024: 228 us without, 197 with.)
  const int rest = S::BM == 256 ? tiles % CUS : 0, parts = rest == 0 ? 1 : rest * 4 <= CUS ? 4 : rest * 2 <= CUS ? 2 : 1;
  const int whole = parts > 1 ? tiles - rest : tiles;
  const int id = blockIdx.x, before_rest = (whole + 7) / 8 * 8;
  if (id < before_rest) {
    const int tile = tile_of_workgroup(id, whole);
    if (tile < 0) return;
    const RowTile t = all.find(p.groups, width, tile);
    rows_tile<S, BF, FB, MODE>(p, t, t.tm * S::BM, t.tn * S::BN);
    return;
  }
  if constexpr (S::BM == 256) {
    const int part = id - before_rest;
    if (parts == 1 || part >= rest * parts) return;
    const RowTile t = all.find(p.groups, width, whole + part / parts);
    const int k = part % parts;
    if (parts == 4) rows_tile<Shape<128, 128, 64, 2, 4>, BF, FB, MODE>(p, t, t.tm * 256 + k / 2 * 128, t.tn * 256 + k % 2 * 128);
    else rows_tile<Shape<128, 256, 64, 2, 4>, BF, FB, MODE>(p, t, t.tm * 256 + k * 128, t.tn * 256);
  }
}

// The same for few rows a group, where what counts is how fast the weights of the groups that have any are read.  A workgroup has
// 16 rows by 32 columns (64 where a row of W in memory runs along them, 128 bytes of each at once); its wavefronts share out the
// slabs of K, each with slabs of its own in LDS and no barriers, so that up to 4 x 3 (or 4 x 2) slabs are under way at once, and
// their sums are added in a fixed order at the end.  Reading W bounds it: 256 rows over 64 groups of 2048 x 1024 in 45.5 us, 5.9
// TB/s; with 2 rows of a 1024 x 4096 group, 4.6 us, the one trip to memory.
template <bool BF, int FB, int MODE>
struct FewRows {
  static constexpr int BM = 16, BN = FB == KS ? 64 : 32, BK = 64, WAVES = 4, STAGES = FB == KS ? 2 : 3;
  using A = Slab<KC, BM, BK, 64>;
  using B = Slab<FB, BN, BK, 64>;
  static constexpr int STAGE = (BM + BN) * BK, STRIDE = BN + 4;
  static constexpr int LDS_BYTES = WAVES * STAGES * STAGE * 2;
  static_assert(BM * STRIDE * 4 <= STAGES * STAGE * 2, "a wavefront's sums lie where its slabs were");
};
template <bool BF, int FB, int MODE>
__global__ __launch_bounds__(256, 2) void k_experts_few_rows(RowsArgs p) {
  using F = FewRows<BF, FB, MODE>;
  using A = typename F::A;
  using B = typename F::B;
  const int width = (p.width + F::BN - 1) / F::BN;
  RowTiles<F::BM> all(p.groups);
  const int tile = tile_of_workgroup(blockIdx.x, (int)min(all.total * width, (int64_t)0x7fffff00));
  if (tile < 0) return;
  const RowTile t = all.find(p.groups, width, tile);
  if (t.tm * F::BM >= t.rows) return;
  const Operand a{p.a + t.lo * p.lda, 0, p.lda, t.rows, p.a_direct};
  const Operand b{p.w + t.g * p.w_stride, 0, p.ldw, p.width, p.w_direct};
  const int r0 = t.tm * F::BM, c0 = t.tn * F::BN, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint16_t* const own = lds_of_launch + wave * F::STAGES * F::STAGE;
  A sa;
  B sb;
  sa.init(a, r0, lane);
  sb.init(b, c0, lane);
  v4f acc[F::BN / 16] = {};
  const auto multiply = [&](const uint16_t* s) {
#pragma unroll
    for (int kk = 0; kk < F::BK / 32; ++kk) {
      const v8s fa = A::fragment(s, 0, kk, lane);
#pragma unroll
      for (int j = 0; j < F::BN / 16; ++j) acc[j] = mma<BF>(B::fragment(s + F::BM * F::BK, j * 16, kk, lane), fa, acc[j]);
    }
  };
  // slabs wave, wave + 4, ..
  const int slabs = MODE == ANY ? (p.depth + F::BK - 1) / F::BK : p.depth / F::BK;
  const int n = (slabs - wave + F::WAVES - 1) / F::WAVES;
  const auto column = [&](int i) { return (wave + i * F::WAVES) * F::BK; };
  if constexpr (MODE == ANY) {
    typename A::Fetched va;
    typename B::Fetched vb;
    const auto fetch = [&](int k) {
      if (A::exists(a, r0, k, p.depth)) sa.fetch_whole(a, r0, k, lane, va);
      else A::fetch(a, r0, k, p.depth, lane, va);
      if (B::exists(b, c0, k, p.depth)) sb.fetch_whole(b, c0, k, lane, vb);
      else B::fetch(b, c0, k, p.depth, lane, vb);
    };
    if (n > 0) fetch(column(0));
    for (int i = 0; i < n; ++i) {
      A::put(a, r0, column(i), p.depth, lane, va, own);
      B::put(b, c0, column(i), p.depth, lane, vb, own + F::BM * F::BK);
      if (i + 1 < n) fetch(column(i + 1));
      lds_done();
      multiply(own);
      lds_done();
    }
  } else {
    const auto load = [&](int i) {
      uint16_t* const s = own + i % F::STAGES * F::STAGE;
      sa.load(a, 0, r0, column(i), s, 0);
      sb.template load<true>(b, 0, c0, column(i), s + F::BM * F::BK, 0);
    };
#pragma unroll
    for (int i = 0; i < F::STAGES; ++i)
      if (i < n) load(i);
    for (int i = 0; i < n; ++i) {
      if (i + F::STAGES <= n) loads_left<(A::PER + B::PER) * (F::STAGES - 1)>();
      else loads_done();
      multiply(own + i % F::STAGES * F::STAGE);
      lds_done();
      if (i + F::STAGES < n) load(i + F::STAGES);
    }
    if (slabs * F::BK < p.depth && wave == slabs % F::WAVES) {      // the last slab, which ends inside
      A::load_any(a, r0, slabs * F::BK, p.depth, own, lane);
      B::load_any(b, c0, slabs * F::BK, p.depth, own + F::BM * F::BK, lane);
      lds_done();
      multiply(own);
      lds_done();
    }
  }
  float* const sums = reinterpret_cast<float*>(own);
#pragma unroll
  for (int j = 0; j < F::BN / 16; ++j) *in_lds<v4f>(sums + (lane & 15) * F::STRIDE + j * 16 + 4 * (lane >> 4)) = acc[j];
  __syncthreads();
  if (threadIdx.x >= F::BM * F::BN / 4) return;
  const int r = threadIdx.x / (F::BN / 4), c = threadIdx.x % (F::BN / 4) * 4;
  v4f v = {};
#pragma unroll
  for (int w = 0; w < F::WAVES; ++w)
    v += *in_lds<const v4f>(reinterpret_cast<const float*>(lds_of_launch + w * F::STAGES * F::STAGE) + r * F::STRIDE + c);
  if (r0 + r < t.rows) store4(p.out, p.out_dtype, (t.lo + r0 + r) * p.ldo + c0 + c, p.width - c0 - c, v);
}

// weight_grad: out_g = a_g^T b_g, a [rows, height], b [rows, width], out [height, width].  Where the tiles are too few for the card
// each has `parts` workgroups, a share of the group's rows each: their sums go to `partial`, and k_experts_join adds them up.  (The
// last one to arrive adding them up in the same launch was tried: making the others' sums visible across the dies took three
// times as long as all the rest, 94 us in place of 33 without parts.)  Both operands are read across their rows in LDS.  Bounded by
// the matrix instructions, 32768 rows over 16 groups of 2048 x 8192 in 1.13 ms, 970 TFLOP/s; with few rows by writing out: 4096 over
// 16 of 512 x 2048, binary32, in 27 us, 2.5 TB/s in one burst.
struct WeightsArgs {
  Groups groups;
  const uint16_t* a;
  const uint16_t* b;
  void* out;
  float* partial;           // [groups * tiles][parts][BM][BN]
  int64_t lda, ldb, out_stride;
  int height, width, out_dtype, accumulate, parts;
  bool a_direct, b_direct;
};
template <class S, bool BF, int MODE>
__global__ __launch_bounds__(S::NT, 2) void k_experts_weights(WeightsArgs p) {
  using P = Product<S, BF, KS, KS, 1, 1, MODE>;
  using R = Results<S>;
  const int nm = (p.height + S::BM - 1) / S::BM, nn = (p.width + S::BN - 1) / S::BN;
  // Each die (tile_of_workgroup) gets an eighth of every group's tiles, whose cost goes with the group's rows.
  const int share = (nm * nn + 7) / 8, all = blockIdx.x >> 3, part = all % p.parts, place = all / p.parts, g = place / share;
  const int t = (blockIdx.x & 7) * share + place % share;
  if (g >= p.groups.n || t >= nm * nn) return;
  int tm, tn, lo, hi;
  tile_in_bands(t, nm, nn, &tm, &tn);
  p.groups.range(g, &lo, &hi);
  const int r0 = tile_start<MODE>(tm, S::BM, p.height), c0 = tile_start<MODE>(tn, S::BN, p.width), row0 = tm * S::BM, col0 = tn * S::BN;
  typename P::Acc acc = {};
  const int each = ((hi - lo + p.parts - 1) / p.parts + S::BK - 1) / S::BK * S::BK, first = lo + part * each, rows = min(each, hi - first);
  if (rows > 0) {
    const Operand a{p.a + first * p.lda, 0, p.lda, p.height, p.a_direct}, b{p.b + first * p.ldb, 0, p.ldb, p.width, p.b_direct};
    P::run(a, b, r0, c0, 0, rows, lds_of_launch, acc);
  } else if (p.accumulate && p.parts == 1) {
    return;
  }
  if constexpr (S::BM == 64) {      // (larger tiles are not split)
    if (p.parts > 1) {
      float* const sums = p.partial + ((int64_t)(g * nm * nn + t) * p.parts + part) * (S::BM * S::BN);
      R::by_rows(acc, lds_of_launch, [&](int r, int c, v4f v) { *reinterpret_cast<v4f*>(sums + r * S::BN + c) = v; });
      return;
    }
  }
  if (!p.accumulate) {
    void* const out = static_cast<char*>(p.out) + g * p.out_stride * (p.out_dtype == F32 ? 4 : 2);
    store_tile<S, BF>(acc, lds_of_launch, out, p.out_dtype, p.width, r0, c0, p.height, p.width, row0, col0);
    return;
  }
  float* const sums = static_cast<float*>(p.out) + g * p.out_stride;
  R::visit(acc, lds_of_launch, [&](const float* own, int tr, int tc) {
    const auto mine = [&](int r, int c) { return r >= row0 && r < p.height && c + 3 >= col0; };
    R::template pass<true>(
        own, r0 + tr, c0 + tc,
        [&](int r, int c) { return mine(r, c) ? load4(sums, F32, (int64_t)r * p.width + c, p.width - c) : v4f{}; },
        [&](int r, int c, v4f v, v4f before) {
          if (mine(r, c)) store_from(sums, (int64_t)r * p.width + c, p.width - c, col0 - c, v + before);
        });
  });
}

// The parts' sums, in their order.  A workgroup a tile.
template <bool BF, int MODE>
__global__ __launch_bounds__(BLOCK) void k_experts_join(WeightsArgs p) {
  constexpr int N = 64;
  const int nm = (p.height + N - 1) / N, nn = (p.width + N - 1) / N, g = blockIdx.x / (nm * nn);
  int tm, tn;
  tile_in_bands(blockIdx.x - g * nm * nn, nm, nn, &tm, &tn);
  const int r0 = tile_start<MODE>(tm, N, p.height), c0 = tile_start<MODE>(tn, N, p.width), row0 = tm * N, col0 = tn * N;
  const float* const sums = p.partial + (int64_t)blockIdx.x * p.parts * (N * N);
#pragma unroll
  for (int u = 0; u < N * N / 4 / BLOCK; ++u) {
    const int k = threadIdx.x + u * BLOCK, r = r0 + k / (N / 4), c = c0 + k % (N / 4) * 4;
    if (r < row0 || r >= p.height || c + 3 < col0 || c >= p.width) continue;
    const int64_t at = g * p.out_stride + (int64_t)r * p.width + c;
    v4f v = {};
    for (int j = 0; j < p.parts; ++j) v += *reinterpret_cast<const v4f*>(sums + j * (N * N) + k * 4);
    if (p.accumulate) v += load4(p.out, F32, at, p.width - c);
    if (p.out_dtype == F32) {
      store_from(p.out, at, p.width - c, col0 - c, v);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c + e >= col0 && c + e < p.width) static_cast<uint16_t*>(p.out)[at + e] = to_bits(v[e], BF);
    }
  }
}

// ---- orthogonalised update -----------------------------------------------------------------------------------------
// Working matrices hold X * 2^12 and S, Y * 2^12, E and B * 2^8 (and Q times a power of two for what the coefficients can
// make of it), so that second terms of common elements are normal binary16 numbers: X's elements are about 1 / sqrt(m n) and
// S's 1 / m at first.
constexpr float X_UNIT = 4096.0f, S_UNIT = 4096.0f, E_UNIT = 256.0f;

// v as a sum of two binary16 numbers.  Both have to come from the same binary32 number: left to itself the compiler may form the
// first from a product before that is rounded to binary32 (v_fma_mixlo_f16), and the second from the rounded one, which puts
// the sum off by 2^-11 for a value close to the middle between two binary16 numbers.
__device__ __forceinline__ void split4(v4f v, v4h* hi, v4h* lo) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float x = v[e];
    asm("" : "+v"(x));
    const _Float16 h = (_Float16)x;
    (*hi)[e] = __builtin_bit_cast(unsigned short, h);
    (*lo)[e] = __builtin_bit_cast(unsigned short, (_Float16)(x - (float)h));
  }
}
template <int TERMS>
__device__ __forceinline__ void store_terms(uint16_t* plane, int64_t term, int64_t at, v4f v) {
  v4h hi, lo;
  split4(v, &hi, &lo);
  *reinterpret_cast<v4h*>(plane + at) = hi;
  if constexpr (TERMS == 2) *reinterpret_cast<v4h*>(plane + term + at) = lo;
}

template <int TERMS>
__device__ __forceinline__ void store_terms8(uint16_t* plane, int64_t term, int64_t at, v4f a, v4f b) {
  v4h ha, la, hb, lb;
  split4(a, &ha, &la);
  split4(b, &hb, &lb);
  typedef unsigned short v8u __attribute__((ext_vector_type(8)));
  *reinterpret_cast<v8u*>(plane + at) = __builtin_shufflevector(ha, hb, 0, 1, 2, 3, 4, 5, 6, 7);
  if constexpr (TERMS == 2) *reinterpret_cast<v8u*>(plane + term + at) = __builtin_shufflevector(la, lb, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Two ways through the Newton-Schulz steps X <- B X, B = a + b S + c S^2, S = X X^T, of which the first two products of three
// are symmetric: half their tiles are computed, each written on both sides of the diagonal.
//
// With 22-bit operands (two terms everywhere) X is left alone and what becomes of S is followed instead: all these matrices
// are polynomials of S, they commute, so that S' = B S B and, for several steps together, X' = Q X with Q the product of
// the B: four symmetric products of [m, m] a step (B, Y = B S, S' = Y B, Q' = B Q) in place of one symmetric and one full
// product of [m, n].  A singular value near zero has its square in S, beside rounding errors of the largest one's, and both
// grow by a^2 a step; so S is formed from X again after steps that together make more than 2^8 of it.  The usual 5 steps
// are 3 and 2: of multiply-adds, in m^3, 3 n / m + 7 in place of 7.5 n / m + 2.5, the same for n = m, 19 in place of 32.5
// for n = 4 m.
// In the 2-norm over the matrix 1e-6 to 3e-6 off for matrices of normal numbers, 1.6e-5 for a sixteenth of the rank with 1%
// noise (binary32 products in the plain order: 1e-6 to 2e-6, and 1.7e-5); with one S for all 5 steps 3e-5 and 2e-3.
//
// With 11 bits for the [m, m] matrices those errors would be 1e-1, so there the plain order stays: with c != 0,
// a + b S + c S^2 = c E^2 + d, E = S - t, t = -b / 2c, d = a - b^2 / 4c, one product E E^T and nothing to read beside it, and
// where the singular values end up (S near 1) E is small, and so is what its rounding costs.  A c that is small beside b would
// put t, and with it E's rounding errors, far beyond S; outside of [0, 2], which S ends in the middle of, t is 1 and E is read
// once more for the term that is left, (b + 2 c t) E.  X keeps two terms: rounding it to 11 bits would drown the small singular
// vectors of a matrix of low rank (3e-2 in place of 2e-3).
struct Shifted {      // a + b S + c S^2 = c E^2 + linear E + constant, E = S - t
  float t, linear, constant;
};
__host__ __device__ inline Shifted shifted(float a, float b, float c) {
  const double vertex = -(double)b / (2.0 * c);
  const bool there = vertex >= 0.0 && vertex <= 2.0;
  const double t = there ? vertex : 1.0;
  return Shifted{(float)t, there ? 0.0f : (float)(b + 2.0 * c * t), (float)(a + t * (b + c * t))};
}

// One or two products of [mp, mp] results over the list, of which those with j == blockIdx.y: out = mul A B^T + add_mul ADD +
// diag on the diagonal.  48 matrices with m = 1024, 22 bits, half their tiles: X X^T with n = 4096 in 637 us (P), 1210 TFLOP/s of
// matrix instructions, which bound it; the products 1024 deep in 226 us (P), 850 TFLOP/s, the matrix units busy half the time: the
// results, on both sides of the diagonal, are written by all CUs at about the same time.
struct SymmetricArgs {
  const ListTile* tiles;
  const uint16_t* a;           // X, or [mp, mp]
  const uint16_t* b[2];
  const uint16_t* add;         // NULL: none; else added to the first
  uint16_t* out[2];
  int64_t x_term, term;
  float mul[2], add_mul, diag;
};
template <class S, int TERMS, bool FROM_X>
__global__ __launch_bounds__(S::NT, 2) void k_polar_symmetric(SymmetricArgs p) {
  using P = Product<S, false, KC, KC, TERMS, TERMS, WHOLE>;
  using R = Results<S>;
  const ListTile t = p.tiles[blockIdx.x];
  if (t.mp == 0) return;
  const int mp = t.mp, which = blockIdx.y;
  typename P::Acc acc = {};
  const int tr = t.tm * S::BM, tc = t.tn * S::BN;
  if constexpr (FROM_X) {
    const Operand x{p.a + t.x, p.x_term, t.np, mp, true};
    P::run(x, x, tr, tc, 0, t.np, lds_of_launch, acc);
  } else {
    const Operand a{p.a + t.e, p.term, mp, mp, true}, b{p.b[which] + t.e, p.term, mp, mp, true};
    P::run(a, b, tr, tc, 0, mp, lds_of_launch, acc);
  }
  uint16_t* const out = p.out[which] + t.e;
  const uint16_t* const add = which == 0 && p.add ? p.add + t.e : nullptr;
  const float mul = p.mul[which], diag = which == 0 ? p.diag : 0.0f;
  // Element (r + e dr, c + e dc) is element e of the eight from (r, c) on; all of them lie in a row of `out` (and of ADD), turned over
  // the diagonal where dr is 1.
  const auto half = [&](const float* own, int r0, int c0, auto rowwise) {
    constexpr int dr = rowwise ? 0 : 1, dc = rowwise ? 1 : 0;
    const auto at = [&](int r, int c) { return rowwise ? (int64_t)(tr + r) * mp + tc + c : (int64_t)(tc + c) * mp + tr + r; };
    const auto inside = [&](int r, int c) { return tr + r < mp && tc + c < mp; };
    using Eight = typename R::Eight;
    R::template pass8<rowwise>(
        own, r0, c0,
        [&](int r, int c) {
          Eight v = {};
          if (add && inside(r, c)) {
            const v8s hi = *reinterpret_cast<const v8s*>(add + at(r, c));
            v8s lo = {};
            if constexpr (TERMS == 2) lo = *reinterpret_cast<const v8s*>(add + p.term + at(r, c));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              v.a[e] = p.add_mul * (from_bits((unsigned short)hi[e], false) + from_bits((unsigned short)lo[e], false));
              v.b[e] = p.add_mul * (from_bits((unsigned short)hi[e + 4], false) + from_bits((unsigned short)lo[e + 4], false));
            }
          }
          return v;
        },
        [&](int r, int c, Eight v, Eight w) {
          if (!inside(r, c)) return;
          v.a = v.a * mul + w.a;
          v.b = v.b * mul + w.b;
          const int off = (tc + c) - (tr + r);      // (0: the first of the eight is on the diagonal)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (off + e * (dc - dr) == 0) v.a[e] += diag;
            if (off + (e + 4) * (dc - dr) == 0) v.b[e] += diag;
          }
          store_terms8<TERMS>(out, p.term, at(r, c), v.a, v.b);
        });
  };
  R::visit(acc, lds_of_launch, [&](const float* own, int r0, int c0) {
    half(own, r0, c0, std::true_type{});
    if (t.tm != t.tn) half(own, r0, c0, std::false_type{});
  });
}

// What becomes of the last X: out = X in the list's order (orthogonalize), or the update of the parameters.
struct Finish {
  float* x;                 // NULL: orthogonalize
  void* out;                // x_lp (or NULL), or the orthogonaliser's output
  int dtype;
  float lr, keep;           // keep = 1 - lr * weight_decay
};

// X' = mul B X, or with LAST what becomes of it.  Bounded as the symmetric products: 48 of [1024, 1024] by [1024, 4096], 22 bits,
// in 1.03 ms (P), 1200 TFLOP/s of matrix instructions; with the update of binary32 parameters 1.34 ms (P).
struct ApplyArgs {
  const ListTile* tiles;
  const Matrix* mats;
  const uint16_t* b;
  const uint16_t* x;
  uint16_t* out;
  int64_t b_term, x_term;
  float mul;
  Finish finish;
};
template <class S, int B_TERMS, bool LAST>
__global__ __launch_bounds__(S::NT, 2) void k_polar_apply(ApplyArgs p) {
  using P = Product<S, false, KC, KS, B_TERMS, 2, WHOLE>;
  using R = Results<S>;
  const ListTile t = p.tiles[blockIdx.x];
  if (t.mp == 0) return;
  typename P::Acc acc = {};
  const Operand a{p.b + t.e, p.b_term, t.mp, t.mp, true}, b{p.x + t.x, p.x_term, t.np, t.np, true};
  const int tr = t.tm * S::BM, tc = t.tn * S::BN;
  P::run(a, b, tr, tc, 0, t.mp, lds_of_launch, acc);
  if constexpr (!LAST) {
    using Eight = typename R::Eight;
    R::visit(acc, lds_of_launch, [&](const float* own, int r0, int c0) {
      R::template pass8<true>(
          own, tr + r0, tc + c0, [](int, int) { return Eight{}; },
          [&](int r, int c, Eight v, Eight) {
            if (r < t.mp && c < t.np) store_terms8<2>(p.out + t.x, p.x_term, (int64_t)r * t.np + c, v.a * p.mul, v.b * p.mul);
          });
    });
  } else {
    const Matrix& m = p.mats[t.mat];
    const int rows = m.rows, cols = m.cols;
    const int64_t base = m.at;
    const float step = p.finish.lr * m.scale, mul = p.mul * (1.0f / X_UNIT);
    // A tall matrix's X is its transpose: what is a column there is part of a row of the list's matrix.
    const auto rows_of = [&](const float* own, int r0, int c0, auto rowwise) {
      const auto row = [&](int r, int c) { return rowwise ? tr + r : tc + c; };
      const auto col = [&](int r, int c) { return rowwise ? tc + c : tr + r; };
      R::template pass<rowwise>(
          own, r0, c0,
          [&](int r, int c) {
            if (!p.finish.x || row(r, c) >= rows) return v4f{};
            return load4(p.finish.x, F32, base + (int64_t)row(r, c) * cols + col(r, c), cols - col(r, c));
          },
          [&](int r, int c, v4f v, v4f x) {
            if (row(r, c) >= rows) return;
            const int64_t at = base + (int64_t)row(r, c) * cols + col(r, c);
            const int left = cols - col(r, c);
            v4f o = v * mul;
            if (p.finish.x) {
#pragma unroll
              for (int e = 0; e < 4; ++e) o[e] = x[e] * p.finish.keep - step * o[e];
              store4(p.finish.x, F32, at, left, o);
            }
            if (p.finish.out) store4(p.finish.out, p.finish.dtype, at, left, o);
          });
    };
    R::visit(acc, lds_of_launch, [&](const float* own, int r0, int c0) {
      if (m.tall) rows_of(own, r0, c0, std::false_type{});
      else rows_of(own, r0, c0, std::true_type{});
    });
  }
}

// Element-wise tiles are SIDE x SIDE elements of a matrix in the list's order, padding included; a thread has four
// adjacent elements of rows t / 16 + 16 j.
struct SquareTile {
  int mat, row0, col0;
};

// The direction u of a step, from m after its update.
struct Direction {
  const void* g;     // NULL: m itself
  const float* m;    // NULL: g itself (orthogonalize)
  int dtype, nesterov;
  float scale, beta, omb;
};
__device__ __forceinline__ v4f direction4(const Direction& d, v4f g, v4f m) {
  if (!d.m) return g;
  if (!d.g || !d.nesterov) return m;
  v4f u;
#pragma unroll
  for (int e = 0; e < 4; ++e) u[e] = d.beta * m[e] + d.omb * (d.scale * g[e]);
  return u;
}

// m <- beta m + (1 - beta) scale g, and the sum of u's squares over each tile, in binary64.  Bounded by HBM: 302M elements with
// binary32 gradients in 670 us (P), 5.4 TB/s.
__global__ __launch_bounds__(BLOCK) void k_muon_moments(const SquareTile* tiles, const Matrix* mats, Direction d, float* m_out, double* sums) {
  const SquareTile t = tiles[blockIdx.x];
  const Matrix& mat = mats[t.mat];
  double s = 0.0;
#pragma unroll
  for (int j = 0; j < SIDE / 16; ++j) {
    const int r = t.row0 + threadIdx.x / 16 + 16 * j, c = t.col0 + threadIdx.x % 16 * 4;
    if (r >= mat.rows || c >= mat.cols) continue;
    const int64_t at = mat.at + (int64_t)r * mat.cols + c;
    const int left = mat.cols - c;
    v4f g = {}, m = {};
    if (d.g) g = load4(d.g, d.dtype, at, left);
    if (d.m) m = load4(d.m, F32, at, left);
    if (d.m && d.g) {
#pragma unroll
      for (int e = 0; e < 4; ++e) m[e] = d.beta * m[e] + d.omb * (d.scale * g[e]);
      store4(m_out, F32, at, left, m);
    }
    const v4f u = direction4(d, g, m);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) s += (double)u[e] * (double)u[e];
  }
  __shared__ double part[BLOCK / 64];
#pragma unroll
  for (int k = 32; k; k >>= 1) s += __shfl_xor(s, k);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) sums[blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

// X_UNIT / (norm + eps) as two factors: their product need not be a normal binary32 number, the first is a power of two that makes the
// second one, and 1 for all but the smallest and the largest of norms.
struct Inverse {
  float first, second;
};
__device__ __forceinline__ Inverse inverse_of(double squares, float eps) {
  const double d = sqrt(squares) + (double)eps;
  const float first = d < 0x1p-100 ? 0x1p100f : d > 0x1p130 ? 0x1p-30f : 1.0f;
  return Inverse{first, (float)((double)X_UNIT / (d * (double)first))};
}
// That of a matrix, in every thread of a workgroup
__device__ __forceinline__ Inverse inverse_norm(const Matrix& m, const double* sums, float eps) {
  double s = 0.0;
  for (int i = threadIdx.x; i < m.tiles; i += BLOCK) s += sums[m.tile0 + i];
  __shared__ double part[BLOCK / 64];
#pragma unroll
  for (int k = 32; k; k >>= 1) s += __shfl_xor(s, k);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  return inverse_of((part[0] + part[1]) + (part[2] + part[3]), eps);
}
__global__ __launch_bounds__(BLOCK) void k_muon_norms(const Matrix* mats, const double* sums, float eps, Inverse* inv) {
  const Inverse f = inverse_norm(mats[blockIdx.x], sums, eps);
  if (threadIdx.x == 0) inv[blockIdx.x] = f;
}

// X = u / (norm + eps), transposed for tall matrices, zeros around it.  inv == NULL: every workgroup adds up its matrix's sums
// itself, which for matrices of few tiles takes less than a launch (norms_apart).  Bounded by HBM: 302M elements of m and g into two
// terms in 700 us (P), 5.2 TB/s.
__global__ __launch_bounds__(BLOCK) void k_muon_pack(const SquareTile* tiles, const Matrix* mats, Direction d, const Inverse* inv, const double* sums,
                                                     float eps, uint16_t* x, int64_t term) {
  __shared__ float turned[SIDE][SIDE + 1];
  const SquareTile t = tiles[blockIdx.x];
  const Matrix& mat = mats[t.mat];
  const Inverse f = inv ? inv[t.mat] : inverse_norm(mat, sums, eps);
#pragma unroll
  for (int j = 0; j < SIDE / 16; ++j) {
    const int y = threadIdx.x / 16 + 16 * j, z = threadIdx.x % 16 * 4, r = t.row0 + y, c = t.col0 + z;
    v4f v = {};
    if (r < mat.rows && c < mat.cols) {
      const int64_t at = mat.at + (int64_t)r * mat.cols + c;
      const int left = mat.cols - c;
      v4f g = {}, m = {};
      if (d.g && (!d.m || d.nesterov)) g = load4(d.g, d.dtype, at, left);
      if (d.m) m = load4(d.m, F32, at, left);
      const v4f u = direction4(d, g, m);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = e < left ? u[e] * f.first * f.second : 0.0f;
    }
    if (!mat.tall) {
      store_terms<2>(x + mat.x, term, (int64_t)r * mat.np + c, v);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) turned[z + e][y] = v[e];
    }
  }
  if (!mat.tall) return;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < SIDE / 16; ++j) {
    const int y = threadIdx.x / 16 + 16 * j, z = threadIdx.x % 16 * 4;
    const v4f v = {turned[y][z], turned[y][z + 1], turned[y][z + 2], turned[y][z + 3]};
    store_terms<2>(x + mat.x, term, (int64_t)(t.col0 + y) * mat.np + t.row0 + z, v);
  }
}

// A whole list of small matrices (m <= 64, n <= 512) in one launch, a workgroup each: X stays in LDS as two terms from the
// gradient to the updated parameters, step by step with 22 bits (in both precisions: it is not the multiply-adds that
// count here, but the fifteen products' latency).  12 matrices of 64 x 64 to 256 x 64 with momentum and update: 41 us, of
// which about 17 are the way in and out, in trips to memory that wait for each other; a step takes 2.8 us and 0.6 for every 64 columns more (its
// binary16 pairs cost as much as its products).  74 us with tiles, and less than those at every size measured, us in one launch /
// with tiles of 22 bits / of 11: 12 of 64 x 64 19 / 61 / 56, 12 of 64 x 512 62 / 78 / 66, one of it 61 / 73 / 61, 2048 of 64 x 64 99 / 243 / 188,
// 2048 of 64 x 512 595 / 821 / 954.
constexpr int SMALL_NT = 512, MAX_STEPS = 64;
struct SmallArgs {
  const Matrix* mats;
  Direction d;
  float* m_out;
  Finish finish;
  float eps;
  int steps;
  float coefficients[3 * MAX_STEPS];
};
// X and E in LDS: a row's eights of columns, permuted by the row's number, each 32 bytes: eight first terms and eight second
// ones, or the same eight as binary32 (u at the start, the result at the end).
__device__ __forceinline__ int small_at(int r, int c, int ld) { return r * 2 * ld + ((((c >> 3) ^ (r & 7)) << 4) | (c & 7)); }
__device__ __forceinline__ float* small_f32(uint16_t* a, int r, int c, int ld) {
  return reinterpret_cast<float*>(a + small_at(r, c & ~7, ld)) + (c & 7);
}
__device__ __forceinline__ void small_put4(uint16_t* at, v4f v) {
  v4h hi, lo;
  split4(v, &hi, &lo);
  *in_lds<v4h>(at) = hi;
  *in_lds<v4h>(at + 8) = lo;
}

// The loops are kept short: the code runs a few times only, and what is unrolled has to be fetched first (with everything
// unrolled, 48 KB in place of 14, it took 44 us in place of 41).
__global__ __launch_bounds__(SMALL_NT, 2) void k_polar_small(SmallArgs p) {
  __shared__ double part[SMALL_NT / 64];
  const Matrix& mat = p.mats[blockIdx.x];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, q = lane >> 4;
  const int rows = mat.rows, cols = mat.cols, np = mat.np;
  const bool tall = mat.tall;
  uint16_t* const X = lds_of_launch;                       // [SMALL_M][np]
  uint16_t* const E = lds_of_launch + 2 * SMALL_M * np;    // [SMALL_M][SMALL_M]: E, then B
  // The list's matrix, four elements of a row at a time: piece k is (r, c..c + 3); k advances by SMALL_NT
  const int row_pieces = (cols + 3) / 4, pieces = rows * row_pieces;
  const int step_r = SMALL_NT / row_pieces, step_c = SMALL_NT % row_pieces;

  for (int k = tid; k < SMALL_M * np / 4; k += SMALL_NT) *in_lds<v8s>(X + 8 * k) = v8s{};      // (the padding)
  __syncthreads();
  // u, in binary32, and its norm
  double s = 0.0;
  {
    int r = tid / row_pieces, c4 = tid % row_pieces;
#pragma unroll 2
    for (int k = tid; k < pieces; k += SMALL_NT) {
      const int c = c4 * 4, left = cols - c;
      const int64_t at = mat.at + (int64_t)r * cols + c;
      v4f g = {}, m = {};
      if (p.d.g) g = load4(p.d.g, p.d.dtype, at, left);
      if (p.d.m) m = load4(p.d.m, F32, at, left);
      if (p.d.m && p.d.g) {
#pragma unroll
        for (int e = 0; e < 4; ++e) m[e] = p.d.beta * m[e] + p.d.omb * (p.d.scale * g[e]);
        store4(p.m_out, F32, at, left, m);
      }
      v4f u = direction4(p.d, g, m);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (e >= left) u[e] = 0.0f;
        s += (double)u[e] * (double)u[e];
        if (tall && e < left) *in_lds<float>(small_f32(X, c + e, r, np)) = u[e];
      }
      if (!tall) *in_lds<v4f>(small_f32(X, r, c, np)) = u;
      c4 += step_c;
      r += step_r + (c4 >= row_pieces);
      c4 -= c4 >= row_pieces ? row_pieces : 0;
    }
  }
#pragma unroll
  for (int k = 32; k; k >>= 1) s += __shfl_xor(s, k);
  if (lane == 0) part[wave] = s;
  __syncthreads();
  s = 0.0;
#pragma unroll
  for (int k = 0; k < SMALL_NT / 64; ++k) s += part[k];
  const Inverse f = inverse_of(s, p.eps);
  for (int k = tid; k < SMALL_M * np / 8; k += SMALL_NT) {      // eights of X, wherever they are
    uint16_t* const at = X + 16 * k;
    const v4f u0 = *in_lds<const v4f>(at), u1 = *in_lds<const v4f>(at + 8);
    small_put4(at, u0 * f.first * f.second);
    small_put4(at + 4, u1 * f.first * f.second);
  }
  __syncthreads();

  // rows f .. f + 15, columns 32 kk + 8 q + 0..7; `term` 0 or 8
  const auto by_row = [&](const uint16_t* a, int f0, int kk, int ld, int term) {
    return *in_lds<const v8s>(a + small_at(f0 + i, kk * 32 + 8 * q, ld) + term);
  };
  // X's columns f .. f + 15, rows 32 kk + 8 q + 0..7
  const auto by_column = [&](const uint16_t* a, int f0, int kk, int term) {
    const int r = kk * 32 + 8 * q + (i >> 2), c = f0 + (i & 3) * 4;
    const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(in_lds<v4s>(a + small_at(r, c, np) + term));
    const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(in_lds<v4s>(a + small_at(r + 4, c, np) + term));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  // Of [64, 64] a wavefront has 16 rows by 32 columns; lane (q, i) row i, four columns from 4 q on.  Its sums are kept apart
  // by term, so that no product waits for the one before.
  const int er = wave / 2 * 16, ec = wave % 2 * 32;
  v4f acc[2], own[2] = {};      // sums, and of E what this wavefront wrote
  const auto symmetric = [&](const uint16_t* a, int ld) {
    v4f sum[2][3] = {};
    for (int kk = 0; kk < ld / 32; ++kk) {
      const v8s l0 = by_row(a, er, kk, ld, 0), l1 = by_row(a, er, kk, ld, 8);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const v8s r0 = by_row(a, ec + 16 * j, kk, ld, 0), r1 = by_row(a, ec + 16 * j, kk, ld, 8);
        sum[j][0] = mma<false>(r0, l0, sum[j][0]);
        sum[j][1] = mma<false>(r1, l0, sum[j][1]);
        sum[j][2] = mma<false>(r0, l1, sum[j][2]);
      }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[j] = sum[j][0] + (sum[j][1] + sum[j][2]);
  };
  const auto put_e = [&](float mul, float linear, float diag) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int r = er + i, c = ec + j * 16 + 4 * q;
      v4f v = acc[j] * mul;
      if (linear != 0.0f) v += own[j] * linear;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (r == c + e) v[e] += diag;
      own[j] = v;
      small_put4(E + small_at(r, c, SMALL_M), v);
    }
  };

#pragma unroll 1
  for (int k = 0; k < p.steps; ++k) {
    const float a = p.coefficients[3 * k], b = p.coefficients[3 * k + 1], c = p.coefficients[3 * k + 2];
    const bool last = k + 1 == p.steps;
    constexpr float PER_GRAM = E_UNIT / (X_UNIT * X_UNIT);
    symmetric(X, np);
    if (c != 0.0f) {      // E, then B
      const Shifted form = shifted(a, b, c);
      put_e(PER_GRAM, 0.0f, -form.t * E_UNIT);
      __syncthreads();
      symmetric(E, SMALL_M);
      __syncthreads();
      put_e(c / E_UNIT, form.linear, form.constant * E_UNIT);
    } else {
      put_e(b * PER_GRAM, 0.0f, a * E_UNIT);
    }
    __syncthreads();
    // X <- B X, sixteen columns at a time: nobody else reads those
#pragma unroll 1
    for (int f0 = wave * 16; f0 < np; f0 += SMALL_NT / 64 * 16) {
      v8s x[2][2];
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        x[kk][0] = by_column(X, f0, kk, 0);
        x[kk][1] = by_column(X, f0, kk, 8);
      }
      lds_done();
#pragma unroll 2
      for (int t = 0; t < 4; ++t) {
        v4f sum[3] = {};
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
          const v8s b0 = by_row(E, t * 16, kk, SMALL_M, 0), b1 = by_row(E, t * 16, kk, SMALL_M, 8);
          sum[0] = mma<false>(x[kk][0], b0, sum[0]);
          sum[1] = mma<false>(x[kk][1], b0, sum[1]);
          sum[2] = mma<false>(x[kk][0], b1, sum[2]);
        }
        const v4f o = (sum[0] + (sum[1] + sum[2])) * (1.0f / E_UNIT);
        const int r = t * 16 + i, col = f0 + 4 * q;
        if (last) *in_lds<v4f>(small_f32(X, r, col, np)) = o * (1.0f / X_UNIT);
        else small_put4(X + small_at(r, col, np), o);
      }
    }
    __syncthreads();
  }

  const float step = p.finish.lr * mat.scale;
  int r = tid / row_pieces, c4 = tid % row_pieces;
#pragma unroll 2
  for (int k = tid; k < pieces; k += SMALL_NT) {
    const int c = c4 * 4, left = cols - c;
    const int64_t at = mat.at + (int64_t)r * cols + c;
    v4f o;
    if (tall) {
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = *in_lds<const float>(small_f32(X, min(c + e, cols - 1), r, np));
    } else {
      o = *in_lds<const v4f>(small_f32(X, r, c, np));
    }
    if (p.finish.x) {
      const v4f x = load4(p.finish.x, F32, at, left);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = x[e] * p.finish.keep - step * o[e];
      store4(p.finish.x, F32, at, left, o);
    }
    if (p.finish.out) store4(p.finish.out, p.finish.dtype, at, left, o);
    c4 += step_c;
    r += step_r + (c4 >= row_pieces);
    c4 -= c4 >= row_pieces ? row_pieces : 0;
  }
}

}  // namespace obm
