// Host check of the addresses in q4_rows.h: for rows of every small number of
// columns, codes at every distance from a multiple of 4 and every row of a matrix,
// the words that the matrix-product kernel reads behind a step hold a byte of the
// array at least (aligned words of 4 bytes then stay inside its pages), and the one
// that a row's own last bytes in the step need is that one.
#include <cstdint>
#include <cstdio>

#include "q4_rows.h"

int main() {
  using namespace ebag;
  int bad = 0, cases = 0;
  const int step_bytes = 64;  // 128 columns
  for (int64_t K = 1; K <= 700; ++K)
    for (int64_t rows : {1, 2, 3, 33})
      for (uintptr_t at = 4096; at < 4100; ++at) {
        const int64_t row_bytes = (K + 1) / 2, bytes = rows * row_bytes;
        if (row_bytes % 4 == 0 && at % 4 == 0) continue;  // loaded without shifts
        const uint8_t* codes = reinterpret_cast<const uint8_t*>(at);
        const uint8_t* end = codes + bytes;
        const int64_t steps = (K + 127) / 128;
        for (int64_t m = 0; m < rows; ++m)
          for (int64_t s = 0; s < steps; ++s) {
            ++cases;
            const uintptr_t begins = at + m * row_bytes + s * step_bytes;  // the step's first byte
            const uint32_t shift = begins & 3;
            const uint8_t* row = reinterpret_cast<const uint8_t*>(begins - shift);
            const uint8_t* p = word_behind(row, step_bytes, shift, end);
            const uintptr_t q = reinterpret_cast<uintptr_t>(p);
            if (q % 4 || q + 4 <= at || p >= end) ++bad;
            // The step's bytes beyond its 16 whole words, where the row has them.
            const uintptr_t row_end = at + (m + 1) * row_bytes;
            if (shift && begins - shift + step_bytes < row_end && q != begins - shift + step_bytes) ++bad;
          }
      }
  std::printf("cases=%d bad=%d\n", cases, bad);
  return bad != 0;
}
