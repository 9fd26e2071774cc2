// Which kernels the rules of ob_linear8_plan.h choose: ROWS COLS SLABS WIDE EIGHTS a line on standard input, an answer a line:
// "few" and its columns and wavefronts, or the tiles' kind and the number of parts.
#include <cstdio>
#include <cstdlib>
#include <iostream>

#include "ob_linear8_plan.h"

using namespace obl;

int main() {
  long long rows, cols, slabs;
  int wide, eights;
  const char* const names[] = {"W256", "W128", "W64", "TEAMS64", "FLOW256"};
  while (std::cin >> rows >> cols >> slabs >> wide >> eights) {
    if (few8(rows, slabs)) {
      const FewPlan8 p = few_plan8(cols, slabs);
      std::printf("few %d %d\n", p.columns, p.waves);
      continue;
    }
    const Plan8 p = plan8(rows, cols, slabs, wide, eights && slabs >= 2);
    if (p.parts < 1 || p.parts > (slabs > 1 ? slabs : 1) || (p.parts > 1 && (p.kind == FLOW256 || p.parts * rows * cols * 4 > WORKSPACE8))) abort();
    std::printf("%s %d\n", names[p.kind], p.parts);
  }
}
