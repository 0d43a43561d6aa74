// What the products with 4-bit and with 8-bit weights share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tiles.h"

namespace ebag {

// Which rows of y, and whose matrix, slot number `slot` of tiles of `cols` rows
// covers.  Every expert's rows make ceil(n / cols) tiles, in order; the dropped
// rows behind them make tiles of a matrix number `experts`, to be filled with
// zeros.  Found by every wave for itself: 64 experts at once.  false: no tile.
// Args: offsets, experts and rows of the call.
template <class Args>
__device__ __forceinline__ bool find_tile(const Args& a, uint32_t slot, uint32_t cols, int* expert, uint32_t* first,
                                          uint32_t* end) {
  if (!a.offsets) {
    *expert = 0;
    *first = slot * cols;
    *end = a.rows;
    return *first < a.rows;
  }
  const int lane = threadIdx.x & 63;
  uint32_t before = 0;  // tiles of the experts before these 64
  for (int e0 = 0; e0 <= a.experts; e0 += 64) {
    const int e = e0 + lane;
    uint32_t lo = a.rows, hi = a.rows;
    if (e <= a.experts) {
      lo = (uint32_t)a.offsets[e];
      if (e < a.experts) hi = (uint32_t)a.offsets[e + 1];
      lo = lo < a.rows ? lo : a.rows;
      hi = hi < a.rows ? hi : a.rows;
    }
    const uint32_t tiles = hi > lo ? (hi - lo + cols - 1) / cols : 0;
    uint32_t upto = tiles;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const uint32_t v = __shfl_up(upto, d);
      if (lane >= d) upto += v;
    }
    const uint64_t over = __ballot(before + upto > slot);
    if (over) {
      const int at = __builtin_ctzll(over);
      const uint32_t skip = before + __shfl(upto - tiles, at);
      *expert = e0 + at;
      *first = __builtin_amdgcn_readfirstlane(__shfl(lo, at) + (slot - skip) * cols);
      *end = __builtin_amdgcn_readfirstlane(__shfl(hi, at));
      return true;
    }
    before += __shfl(upto, 63);
  }
  return false;
}

// v / (1 + exp(-v)).  With the short exponential, off by (|v| + 8) 2^-22, where y is rounded
// to 16 bits, in two parts below -64, as exp(-v) would overflow where bf16 still holds the
// result (32768 rows on 64 gated experts of 4096 x 2048 in 4 bits 776 -> 784 us); an fp32 y
// gets the full one, of -|v|, which does not overflow where the result is still a number.
template <bool Y32>
__device__ __forceinline__ float silu(float v) {
  if (!Y32) return v / (1.f + __expf(-__builtin_fmaxf(v, -64.f))) * __expf(__builtin_fminf(v + 64.f, 0.f));
  const float e = expf(-fabsf(v));
  return v * ((v < 0.f ? e : 1.f) / (1.f + e));
}

}  // namespace ebag
