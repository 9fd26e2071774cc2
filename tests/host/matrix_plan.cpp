// Which kernels the rules of ob_matrix_plan.h choose: a question a line on standard input, an answer a line.
//   rows GROUPS ROWS DEPTH WIDTH DIRECT              -> "few" or the tiles' kind
//   weights GROUPS ROWS HEIGHT WIDTH MAX_ROWS DIRECT -> kind parts
//   list FINE STEPS (a b c)*STEPS MATRICES (m n)*MATRICES -> of each part: "follow" or "step", terms, kinds of the symmetric and of the full
//                                                            products; or "small"
#include <cstdio>
#include <cstdlib>
#include <iostream>
#include <set>
#include <sstream>
#include <string>
#include <tuple>

#include "ob_matrix_plan.h"

using namespace obm;

// Each tile of each matrix once, of symmetric products those on and above the diagonal; the table's other places are empty
static void check_tiles(const std::vector<Matrix>& mats, const Part& part, ProductKind product) {
  const int side = side_of(product == APPLY ? part.apply_tile : part.sym_tile);
  std::set<std::tuple<int, int, int>> want, found;
  for (const int i : part.list)
    for (int r = 0; r * side < mats[i].mp; ++r)
      for (int c = product == APPLY ? 0 : r; c * side < (product == APPLY ? mats[i].np : mats[i].mp); ++c) want.insert({i, r, c});
  for (const ListTile& t : part.tiles[product]) {
    if (t.mp == 0) continue;
    if (!found.insert({t.mat, t.tm, t.tn}).second || t.mp != mats[t.mat].mp || t.np != mats[t.mat].np) abort();
  }
  if (found != want || part.tiles[product].size() % 8) abort();
}

int main() {
  const char* const names[KINDS] = {"T256", "T128", "T64", "DEEP"};
  std::string line, what;
  while (std::getline(std::cin, line)) {
    std::istringstream in(line);
    in >> what;
    if (what == "rows") {
      int64_t groups, rows, depth, width;
      bool direct;
      in >> groups >> rows >> depth >> width >> direct;
      const RowsPlan p = rows_plan(groups, rows, depth, width, direct);
      printf("%s\n", p.few ? "few" : names[p.kind]);
    } else if (what == "weights") {
      int64_t groups, rows, max_rows;
      int height, width;
      bool direct;
      in >> groups >> rows >> height >> width >> max_rows >> direct;
      const WeightsPlan p = weights_plan(groups, rows, height, width, most_parts(groups, height, width, max_rows), direct);
      printf("%s %d\n", names[p.kind], p.parts);
    } else {
      bool fine;
      int steps, count;
      in >> fine >> steps;
      std::vector<float> coefficients((size_t)(3 * steps));
      for (float& c : coefficients) in >> c;
      in >> count;
      std::vector<Matrix> mats;
      int largest_m = 0, largest_n = 0;
      for (int i = 0; i < count; ++i) {
        Matrix m{};
        in >> m.mp >> m.np;
        m.mp = (m.mp + SIDE - 1) / SIDE * SIDE;
        m.np = (m.np + SIDE - 1) / SIDE * SIDE;
        largest_m = std::max(largest_m, m.mp);
        largest_n = std::max(largest_n, m.np);
        mats.push_back(m);
      }
      if (largest_m <= SMALL_M && largest_n <= SMALL_N) {
        printf("small\n");
        continue;
      }
      for (const Part& p : parts_of(mats, coefficients, fine)) {
        for (const ProductKind k : {GRAM, SYMMETRIC, APPLY}) check_tiles(mats, p, k);
        printf("%s %d %s %s  ", p.follow_s ? "follow" : "step", p.terms, names[p.sym_tile], names[p.apply_tile]);
      }
      printf("\n");
    }
    if (!in) return 1;
  }
}
