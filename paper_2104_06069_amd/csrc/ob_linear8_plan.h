// Host planning of the products in 8 bits (include/ob_layer.h), without any HIP call: which tiles a call takes and how many
// workgroups share a tile's sum, by rules on sizes.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstdint>

namespace obl {

constexpr int CUS8 = 256;                              // of an MI355X
constexpr int64_t WORKSPACE8 = (int64_t)32 << 20;      // bytes of partial sums

// Tiles of 256 x 256 (eight wavefronts, one workgroup on a CU), 128 x 128 and 64 x 64 (four).  TEAMS64: 64 x 64 with eight, four for
// every second slab.  FLOW256: 256 x 256 by workgroups that stay
// (Flow8), for results that it can store.
enum { W256, W128, W64, TEAMS64, KINDS8, FLOW256 = KINDS8 };
constexpr int side8(int kind) { return kind == W256 || kind == FLOW256 ? 256 : kind == W128 ? 128 : 64; }

// What a CU takes for as many tiles of a kind as it runs at once, in microseconds: `fixed` for loading the first slabs and for
// the results, and for each slab of K with all of them, or with one alone.  Measured at 512 to 4096 rows and columns by 1024 to
// 4096, for 16-bit and for binary32 results.  Two teams against one, where each tile has a CU to itself, 2048 x 512 by 4096: 11.7 / 14.8
// and 16.4 / 19.2 us; where there are two on each, 4096 x 512 by 2048: 14.0 / 10.2 and 18.8 / 15.5.
struct Rate8 {
  int per_cu;
  double fixed, all, one;
};
constexpr Rate8 RATES8[2][KINDS8] = {{{1, 5.3, 1.80, 1.60}, {2, 3.8, 1.00, 0.65}, {3, 3.8, 0.55, 0.32}, {1, 5.0, 0.20, 0.20}},
                                     {{1, 8.3, 3.30, 2.82}, {2, 4.7, 1.75, 1.00}, {3, 3.5, 0.89, 0.53}, {1, 4.6, 0.385, 0.385}}};
inline double tiles_time8(int kind, bool wide, double tiles, double slabs) {
  // (a tile after the other: 16384 x 8192 by 2048 226 us, 8192^3 417 us; 32 tiles alone, 2048 deep, 23.7 us; binary32 results: 8192 x 2048 by
  // 32768 675 us, 32768 x 8192 by 2048 800, alone 47.2)
  if (kind == FLOW256) {
    const double full = std::min(tiles / CUS8, 1.0), rounds = std::ceil(tiles / CUS8);
    return wide ? 8.0 + rounds * (8.0 + slabs * (2.26 + 0.35 * full)) : 6.0 + rounds * (1.9 + slabs * (1.1 + 0.48 * full));
  }
  const Rate8& r = RATES8[wide][kind];
  const double a_cu = std::ceil(tiles / CUS8), rounds = std::floor(a_cu / r.per_cu), rest = a_cu - rounds * r.per_cu;
  const double last = rest > 0 ? r.fixed + slabs * (r.one + (r.all - r.one) * (rest - 1) / std::max(r.per_cu - 1, 1)) : 0.0;
  return rounds * (r.fixed + slabs * r.all) + last;
}

struct Plan8 {
  int kind, parts;      // parts: workgroups that share a tile's slabs of K
};

// Few rows: k_product8_few, whose workgroups have all of the rows and 16 or 32 columns, and read all of the rows each.  Microseconds
// with it / with tiles, 16-bit results, the host's call of 6.2 included: 1 row of 8192 x 2048 6.2 / 6.8, 32 rows 6.6 / 6.9, 33 rows 10.2 / 7.9; 1 row
// of 2048 x 8192 7.0 / 9.2, 8 rows 9.2 / 9.9, 16 rows 11.2 / 10.3, 32 rows 16.6 / 11.0; 4 rows of 8192 x 8192 14.1 / 14.8, 8 rows 16.2 / 14.9 (binary32: 16.9 /
// 18.1).  A long K alone, shared by 16 wavefronts at most: 1 row of 512 x 16384 11.4 / 10.6, of 1024 x 65536 40 / 19.
constexpr bool few8(int64_t rows, int64_t slabs) { return rows <= 32 && rows * slabs <= 512 && slabs < 128; }
struct FewPlan8 {
  int columns, waves;      // 16 or 32; 8 or 16
};
inline FewPlan8 few_plan8(int64_t cols, int64_t slabs) {
  if (cols >= 32 * CUS8 && slabs < 64) return FewPlan8{32, 8};
  return FewPlan8{16, slabs > 16 ? 16 : 8};
}

// The kind and number of parts that take the shortest.  Adding parts up is a launch more, reads that wait for each other, and their bytes' way
// to memory and back.  With parts / without, us: 512 x 512 by 8192 12 / 17.6, 128 x 128 by 32768 (16 parts) 14.5 / over 34; 256 x 512 by 2048 8.6 / 6.9.
inline Plan8 plan8(int64_t rows, int64_t cols, int64_t slabs, bool wide, bool flow) {
  Plan8 best{W64, 1};
  double least = 1e300;
  for (int kind = 0; kind < KINDS8 + flow; ++kind) {
    const double tiles = (double)((rows + side8(kind) - 1) / side8(kind)) * (double)((cols + side8(kind) - 1) / side8(kind));
    for (int64_t parts = 1; parts == 1 || (kind != FLOW256 && parts <= slabs / 2 && parts <= 64 && tiles * parts <= 4 * CUS8 && parts * rows * cols * 4 <= WORKSPACE8); parts *= 2) {
      const double join = parts > 1 ? 2.0 + 0.25 * (double)parts + (double)(rows * cols) * 4 * (double)(parts + 1) / 5e6 : 0.0;
      const double t = tiles_time8(kind, wide, tiles * parts, (double)((slabs + parts - 1) / parts)) + join;
      if (t < least) {
        least = t;
        best = Plan8{kind, (int)parts};
      }
    }
  }
  return best;
}

}  // namespace obl
