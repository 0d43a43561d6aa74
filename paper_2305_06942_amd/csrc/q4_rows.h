// Where rows of 4-bit codes lie (host and device, so that the addresses can be
// checked without a GPU).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ebag {

// Rows of codes that begin `shift` bytes behind a multiple of 4 are loaded in aligned
// words and shifted: a step of `bytes` bytes, whose first byte is in the word at `row`,
// needs the word behind its last whole one, too.  It lies at row + bytes, or, where a row
// begins on a multiple of 4 and none is needed, is the last whole one.  In a row's
// last step that may be behind the last matrix, which ends before `end`; the
// step's own bytes then end before it, and its first word, which always holds one
// of them, stands in for it.
__host__ __device__ inline const uint8_t* word_behind(const uint8_t* row, int bytes, uint32_t shift, const uint8_t* end) {
  const uint8_t* p = row + (bytes - (shift ? 0 : 4));
  return p < end ? p : row;
}

}  // namespace ebag
