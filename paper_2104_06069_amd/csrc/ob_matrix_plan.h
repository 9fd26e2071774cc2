// Host planning of the matrix operators (include/ob_matrix.h), without any HIP call or device type: which kernel and which tiles a call
// takes, by rules on sizes, types and alignment, and the tables of tiles of a list's products.  Plain C++, so that the rules can
// be checked on their own.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <vector>

namespace obm {

constexpr int CUS = 256;        // of an MI355X
constexpr int SIDE = 64;        // side of the element-wise kernels' tiles, and what the sides of the working matrices are multiples of

// Tiles of the products: 256 x 256 (eight wavefronts, one workgroup on a CU), 128 x 128 and 64 x 64 (four).  Slabs of 64
// columns, or with two terms of 32: the same LDS.  DEEP: 64 x 64 with two teams of wavefronts, slabs of 64 columns and 128 KB of
// them, for launches of which a CU has one workgroup at most.
enum TileKind { T256, T128, T64, DEEP, KINDS };
constexpr int side_of(int kind) { return kind == T256 ? 256 : kind == T128 ? 128 : 64; }

// What a CU takes for as many tiles of a kind as it runs at once, in microseconds: `fixed` for loading the first slabs and for
// the results, and for each column of K with all of them, or with one alone.  Measured at 8192 x 8192 by 512 to 8192, bfloat16.
struct Rate {
  int per_cu;
  double fixed, all, one;
};
constexpr Rate RATES[KINDS] = {{1, 5.5, 0.0251, 0.0251}, {2, 3.6, 0.0155, 0.0095}, {3, 1.8, 0.0100, 0.0055}, {1, 1.8, 0.0050, 0.0050}};
// Time of `tiles` tiles of the given mean depth, if they are dealt evenly
inline double tiles_time(int kind, double tiles, double depth, bool split_rest = false) {
  const Rate& r = RATES[kind];
  if (split_rest && kind == T256 && tiles > CUS) {      // (k_experts_rows: a last round of up to a quarter or half of the CUs)
    const double rounds = std::floor(tiles / CUS), rest = tiles / CUS - rounds;
    return (r.fixed + depth * r.all) * (rounds + (rest == 0 ? 0.0 : rest <= 0.25 ? 0.4 : rest <= 0.5 ? 0.65 : 1.0));
  }
  const double a_cu = std::ceil(tiles / CUS), rounds = std::floor(a_cu / r.per_cu), rest = a_cu - rounds * r.per_cu;
  const double last = rest > 0 ? r.fixed + depth * (r.one + (r.all - r.one) * (rest - 1) / (r.per_cu - 1)) : 0.0;
  return rounds * (r.fixed + depth * r.all) + last;
}
// The kind whose tiles take the shortest, for `tiles(side)` tiles
template <class F>
int best_tile(F tiles, double depth, bool split_rest = false) {
  int best = T64;
  double least = 1e300;
  for (int kind = 0; kind < KINDS; ++kind) {
    const double t = tiles_time(kind, tiles(side_of(kind)), depth, split_rest);
    if (t < least) {
      least = t;
      best = kind;
    }
  }
  return best;
}

// ---- expert layers -------------------------------------------------------------------------------------------------
// Rows a group (of those that can have one) up to which k_experts_few_rows is taken, and with unaligned operands; us with it / with
// 64 x 64 tiles: 64 rows of 8 experts of 1024 x 1024 8.5 / 13.0, 512 of 32 17.2 / 14.9; 200 of 6 of 555 x 999 8.4 / 11.2
constexpr double FEW_ROWS = 12, FEW_ROWS_ANY = 36;

// Operands that are not `direct` go through registers, for which there are too few beside a 256 x 256 tile's, and no teams
constexpr int kind_of(int kind, bool direct) { return direct ? kind : kind == T256 || kind == T128 ? T128 : T64; }

struct RowsPlan {
  bool few;      // k_experts_few_rows
  int kind;
};
inline RowsPlan rows_plan(int64_t num_groups, int64_t rows, int64_t depth, int64_t width, bool direct) {
  // (a group's last tile is half full in the mean)
  const double groups = (double)std::min(num_groups, rows);
  const int kind = best_tile([&](int n) { return std::max(groups, rows / (double)n + 0.5 * groups) * (double)((width + n - 1) / n); }, (double)depth, true);
  return RowsPlan{rows <= (direct ? FEW_ROWS : FEW_ROWS_ANY) * groups, kind_of(kind, direct)};
}

// weight_grad with more than one workgroup a tile of 64 x 64: the most of them that a context has room for
inline int most_parts(int64_t num_groups, int64_t k, int64_t n, int64_t max_rows) {
  const int64_t tiles = num_groups * ((k + 63) / 64) * ((n + 63) / 64);
  return tiles < 2 * CUS && max_rows >= 256 ? (int)std::min<int64_t>((2 * CUS + tiles - 1) / tiles, 32) : 1;
}
struct WeightsPlan {
  int kind, parts;
};
inline WeightsPlan weights_plan(int64_t num_groups, int64_t rows, int height, int width, int most, bool direct) {
  const auto tiles = [&](int n) { return (double)num_groups * ((height + n - 1) / n) * ((width + n - 1) / n); };
  const double depth = (double)rows / num_groups;
  const int kind = best_tile(tiles, depth);
  // Few tiles of many rows: several workgroups each, as many as fill the card twice and have 128 rows or more.  Adding up
  // takes about 4 us.
  const int parts = (int)std::min({(double)most, std::floor(depth / 128), std::ceil(2 * CUS / tiles(64))});
  if (parts > 1 && 4.0 + tiles_time(T64, tiles(64) * parts, depth / parts) < tiles_time(kind, tiles(side_of(kind)), depth))
    return WeightsPlan{T64, parts};
  return WeightsPlan{kind_of(kind, direct), 1};
}

// ---- orthogonalised update -----------------------------------------------------------------------------------------
// A matrix of the list, and its working matrices: X [mp, np], and those of [mp, mp], binary16, mp and np the sides m <= n
// rounded up to multiples of SIDE.  Zeros around X stay zeros: every product keeps them.
struct Matrix {
  int64_t at;          // in the flat buffers
  int64_t x, e;        // in a plane of X, and of a [mp, mp] matrix
  int rows, cols, mp, np;
  int tall;            // more rows than columns: X is the transpose
  int tile0, tiles;    // its element-wise tiles
  float scale;
};
struct ListTile {      // of a product, with what it needs of its matrix; mp == 0: none
  int64_t x, e;
  int mp, np, mat;
  short tm, tn;
};

constexpr int SMALL_M = 64, SMALL_N = 512;      // k_polar_small (where both sides' times are): lists of which no matrix is larger

// Whether the norms get a launch of their own (k_muon_norms) instead of being added up by every workgroup of k_muon_pack.  us of a call in 11 bits
// with it / without: 4 matrices of 256 tiles 321 / 316, 12 of 256 335 / 327, 4 of 1024 708 / 706, one of 16384 (8192 x 8192) 13753 / 13909,
// (1024 x 65536) 1207 / 1315.
constexpr int NORMS_APART = 256;
inline bool norms_apart(const std::vector<Matrix>& mats) {
  return std::any_of(mats.begin(), mats.end(), [](const Matrix& m) { return m.tiles > NORMS_APART; });
}

// Tiles of a product over the list, dealt to the eight dies: workgroup id runs on die id % 8, so that place id of the table
// is place id / 8 of that die's queue.  Up to 4 x 8 neighbouring tiles of a matrix (what a die runs at once) stay together;
// the dearest go first, each to the queue that has the least to do.
struct Unit {
  double cost;
  int mat, tm0, tm1, tn0, tn1;
};
inline std::vector<ListTile> deal(const std::vector<Matrix>& mats, std::vector<Unit> units, bool upper) {
  std::stable_sort(units.begin(), units.end(), [](const Unit& a, const Unit& b) { return a.cost > b.cost; });
  std::vector<ListTile> queue[8];
  double load[8] = {};
  for (const Unit& u : units) {
    const int q = (int)(std::min_element(load, load + 8) - load);
    for (int tn = u.tn0; tn < u.tn1; ++tn)
      for (int tm = u.tm0; tm < u.tm1; ++tm) {
        if (upper && tn < tm) continue;
        queue[q].push_back(ListTile{mats[u.mat].x, mats[u.mat].e, mats[u.mat].mp, mats[u.mat].np, u.mat, (short)tm, (short)tn});
        load[q] += u.cost;
      }
  }
  size_t longest = 0;
  for (const auto& q : queue) longest = std::max(longest, q.size());
  std::vector<ListTile> table(8 * longest, ListTile{});
  for (int q = 0; q < 8; ++q)
    for (size_t i = 0; i < queue[q].size(); ++i) table[8 * i + q] = queue[q][i];
  return table;
}

enum ProductKind { GRAM, SYMMETRIC, APPLY };
inline std::vector<ListTile> product_tiles(const std::vector<Matrix>& mats, const std::vector<int>& part, int side, ProductKind product) {
  const bool symmetric = product != APPLY;
  std::vector<Unit> units;
  for (const int i : part) {
    const int nm = (mats[i].mp + side - 1) / side, nn = symmetric ? nm : (mats[i].np + side - 1) / side;
    const double cost = (double)(product == GRAM ? mats[i].np : mats[i].mp);
    for (int a = 0; a < nm; a += 4)
      for (int b = 0; b < nn; b += 8) {
        if (symmetric && std::min(b + 8, nn) <= a) continue;
        units.push_back(Unit{cost, i, a, std::min(a + 4, nm), b, std::min(b + 8, nn)});
      }
  }
  return deal(mats, std::move(units), symmetric);
}

inline int product_tile(const std::vector<Matrix>& mats, const std::vector<int>& part, bool symmetric, bool two_terms) {
  double depth = 0, elements = 0;      // of the products' K, weighted by what is computed of them
  for (const int i : part) {
    const double out = symmetric ? 0.5 * mats[i].mp * mats[i].mp : (double)mats[i].mp * mats[i].np;
    depth += out * mats[i].mp;
    elements += out;
  }
  return best_tile([&](int n) {
    double tiles = 0;
    for (const int i : part) {
      const double nm = (mats[i].mp + n - 1) / n, nn = (mats[i].np + n - 1) / n;
      tiles += symmetric ? 0.5 * nm * (nm + 1) : nm * nn;
    }
    return tiles;
  }, (two_terms ? 3.0 : symmetric ? 1.0 : 2.0) * depth / elements);      // products of terms
}

// Steps from k on that follow one S: the growth of a singular value's square up to the last of them (ob_matrix_kernels.h) is at most
// 2^8, or 2^15 where an error of 2e-3 will do.  coefficients: three a step.
inline int steps_from(const std::vector<float>& coefficients, bool fine, int k) {
  const int first = k, steps = (int)coefficients.size() / 3;
  double growth = 1.0;
  for (; k < steps; ++k) {
    if (k > first && growth > (fine ? 256.0 : 32768.0)) break;
    const double a = coefficients[3 * k];
    growth *= std::max(1.0, a * a);
  }
  return k - first;
}

// Matrices that go through the steps together, and the tiles of their products
struct Part {
  bool follow_s = false;      // the way that follows S (ob_matrix_kernels.h); else step by step
  int terms = 2;
  int sym_tile = T64, apply_tile = T64;
  std::vector<int> list;
  // tiles of X X^T, of the other symmetric products (the same ones, but not in the same order: only there depths differ by n)
  // and of B X
  std::vector<ListTile> tiles[3];
  ListTile* d_tiles[3] = {nullptr, nullptr, nullptr};      // ... on the device
};

// Whether following S takes less than going step by step, both with 22 bits, by the tiles' times and LAUNCH a launch
inline bool following_pays(const std::vector<Matrix>& mats, const std::vector<float>& coefficients, const Part& part) {
  constexpr double LAUNCH = 3.0;      // us, from the end of one kernel to the start of the next one's loads
  const int steps = (int)coefficients.size() / 3;
  double depth[3] = {}, out[3] = {};
  for (const int i : part.list)
    for (const ProductKind k : {GRAM, SYMMETRIC, APPLY}) {
      const double n = k == APPLY ? (double)mats[i].mp * mats[i].np : 0.5 * mats[i].mp * mats[i].mp;
      out[k] += n;
      depth[k] += n * (k == GRAM ? mats[i].np : mats[i].mp);
    }
  double t[3];
  for (const ProductKind k : {GRAM, SYMMETRIC, APPLY})
    t[k] = LAUNCH + tiles_time(k == APPLY ? part.apply_tile : part.sym_tile, (double)part.tiles[k].size(), 3.0 * depth[k] / out[k]);
  double followed = 0;
  for (int k = 0, n; k < steps; k += n) {
    n = steps_from(coefficients, true, k);
    followed += t[GRAM] + t[APPLY] + t[SYMMETRIC] * (n + (n - 1)) + (t[SYMMETRIC] - LAUNCH) * 2 * (n - 1) + LAUNCH * n;
  }
  return followed < steps * (t[GRAM] + t[SYMMETRIC] + t[APPLY]);
}

// 11 bits, step by step: 12.5 n / m + 2.5 (in m^3, 5 steps); 22 bits, following S with one S, which will do there: three
// times 1.5 n / m + 8.5, less from n = 3 m on.  With 22 bits following S takes as many multiply-adds as step by step for
// n = m, and more launches and writes (8 of 1024 x 1024: 1010 and 787 us, 4 of 1024 x 4096: 895 and 1277).  Each of the
// two ways is worth launches of its own where there is much for it: MUCH, of m m n, for the wide ones, and with 22 bits for the
// others too.  us apart / together: 22 bits, four [m, m] to one [m, 4 m], 4.3e9 of each 852 / 720 (m = 1024) and 781 / 719 (512),
// 8.6e9 1243 / 1124 and 1263 / 1450, 1.3e10 1601 / 1918, 1.7e10 1990 / 2156 and 2431 / 2829.  11 bits, wide ones following S / all step by
// step: [1024, 4096], 8.6e9 877 / 873 (beside [1024, 1024]), 1.7e10 711 / 594, 5.2e10 1473 / 1531, 2.1e11 5638 / 6014; n = 8 m, 2.6e10
// 726 / 911, 1e11 2008 / 2878; n = 3 m, [768, 2304], 3.3e10 2529 / 2211.  (So at 11 bits n = 3 m and 4 m lose up to a fifth between 1e10 and
// 5e10, and n = 8 m gains as much.)
constexpr double MUCH = 1e10;
inline std::vector<Part> parts_of(const std::vector<Matrix>& mats, const std::vector<float>& coefficients, bool fine) {
  std::vector<int> each[2];
  double work[2] = {};
  for (size_t i = 0; i < mats.size(); ++i) {
    const bool f = mats[i].np >= (fine ? 1.5 : 3.0) * mats[i].mp;
    each[f].push_back((int)i);
    work[f] += (double)mats[i].mp * mats[i].mp * mats[i].np;
  }
  if (work[1] < MUCH || (fine && work[0] < MUCH)) {
    std::vector<int>& all = each[fine];
    all.insert(all.end(), each[!fine].begin(), each[!fine].end());
    each[!fine].clear();
  }
  std::vector<Part> parts;
  for (const int f : {1, 0}) {
    if (each[f].empty()) continue;
    Part part;
    part.list = each[f];
    part.terms = f || fine ? 2 : 1;
    part.sym_tile = product_tile(mats, part.list, true, part.terms == 2);
    part.apply_tile = product_tile(mats, part.list, false, part.terms == 2);
    for (const ProductKind k : {GRAM, SYMMETRIC, APPLY}) part.tiles[k] = product_tiles(mats, part.list, side_of(k == APPLY ? part.apply_tile : part.sym_tile), k);
    part.follow_s = f == 1 && (!fine || following_pays(mats, coefficients, part));
    parts.push_back(std::move(part));
  }
  return parts;
}

}  // namespace obm
