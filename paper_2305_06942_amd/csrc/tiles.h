// Tiles of rows that belong to several experts.
#pragma once

#include <stdint.h>

namespace ebag {

// Most tiles of `cols` rows that `rows` rows of `experts` experts and the
// dropped rows behind them can make.
inline int64_t most_tiles(int64_t rows, int64_t experts, int64_t cols) {
  const int64_t n = (rows + (experts + 1) * (cols - 1)) / cols;
  return n < rows ? n : rows;
}

}  // namespace ebag
