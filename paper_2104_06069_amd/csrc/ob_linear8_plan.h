// Host planning of the products in 8 bits (include/ob_layer.h), without any HIP call: which tiles a call takes and how many
// workgroups share a tile's sum, by rules on sizes.
#pragma once

#include <algorithm>
#include <cstdint>

namespace obl {

constexpr int64_t WORKSPACE8 = (int64_t)32 << 20;      // bytes of partial sums

struct Plan8 {
  int parts;      // workgroups that share a tile's slabs of K
};

inline Plan8 plan8(int64_t rows, int64_t cols, int64_t slabs) {
  const int64_t tiles = ((rows + 63) / 64) * ((cols + 63) / 64);
  // Few tiles of many slabs: several workgroups each, as many as fill the card three times and have eight slabs or more
  const int64_t parts = std::min({(768 + tiles - 1) / tiles, slabs / 8, WORKSPACE8 / 4 / (rows * cols)});
  return Plan8{tiles < 384 && parts > 1 ? (int)parts : 1};
}

}  // namespace obl
