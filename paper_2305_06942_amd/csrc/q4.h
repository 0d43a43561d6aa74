// What the kernels with 4-bit weights share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"
#include "vec16.h"

namespace ebag {

struct Q4Args {
  const uint8_t* codes;
  const char* scales;
  const uint8_t* zeros;     // nullptr: 8
  const char* x;
  char* y;
  const int32_t* offsets;   // nullptr: one matrix, all rows
  const int32_t* src;       // nullptr: row p of x
  int64_t ldx, ldy;         // bytes
  int64_t row_bytes;        // of codes
  int64_t codes_bytes;      // of all matrices
  int64_t M;                // rows of a matrix
  int64_t out_rows;         // of those, the ones a column of y belongs to: M, or M / 2 with glu
  int64_t x_rows;
  uint32_t rows;            // of y
  int32_t K, group, groups;
  int32_t experts;
  int32_t glu;
  int32_t y_f32;
  Divisor by_choices;
  Divisor by_group_blocks;  // group / 32
  Divisor by_tiles;         // tiles of weight rows
};

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// A weight's code q goes through the matrix instructions as 16 + q, which is a
// bit pattern away in fp16 and bf16 (16 is 2^4: q fills the top of the
// mantissa) and exact in both; the 16 and the zero point come off again as
// (16 + zero) * (the sum of x over the group).  fp32 x goes as three bf16
// parts whose sum is x, bit for bit, so its products are exact too.
template <int DT> struct Q4Type;

template <> struct Q4Type<1> {
  static constexpr int PARTS = 1;
  static constexpr uint32_t ONES = 0x3C003C00u;
  // Codes j and j + 4 of a word of eight (low bits first), as 16 + q.
  static __device__ __forceinline__ uint32_t pair(uint32_t w, int j) {
    const uint32_t v = j == 0 ? w << 6 : j == 1 ? w << 2 : j == 2 ? w >> 2 : w >> 6;
    return (v & 0x03C003C0u) | 0x4C004C00u;
  }
  static __device__ __forceinline__ f32x4 mfma(const vec16& a, const vec16& b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};

template <> struct Q4Type<2> {
  static constexpr int PARTS = 1;
  static constexpr uint32_t ONES = 0x3F803F80u;
  static __device__ __forceinline__ uint32_t pair(uint32_t w, int j) {
    const uint32_t v = j == 0 ? w << 3 : j == 1 ? w >> 1 : j == 2 ? w >> 5 : w >> 9;
    return (v & 0x00780078u) | 0x41804180u;
  }
  static __device__ __forceinline__ f32x4 mfma(const vec16& a, const vec16& b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};

template <> struct Q4Type<0> : Q4Type<2> {
  static constexpr int PARTS = 3;
};

// Eight codes of a word in the order of pair(): 0 4, 1 5, 2 6, 3 7.
template <int DT>
__device__ __forceinline__ vec16 unpack_codes(uint32_t w) {
  vec16 r;
#pragma unroll
  for (int j = 0; j < 4; ++j) r[j] = Q4Type<DT>::pair(w, j);
  return r;
}

// Eight consecutive 16-bit elements in that same order.
__device__ __forceinline__ vec16 pair_order(const vec16& v) {
  vec16 r;
  r[0] = __builtin_amdgcn_perm(v[2], v[0], 0x05040100u);
  r[1] = __builtin_amdgcn_perm(v[2], v[0], 0x07060302u);
  r[2] = __builtin_amdgcn_perm(v[3], v[1], 0x05040100u);
  r[3] = __builtin_amdgcn_perm(v[3], v[1], 0x07060302u);
  return r;
}

// Eight consecutive fp32 elements as three vectors of bf16 in pair order: the
// top 8 bits of the significand, the next 8, the last 8 (each cut off, so
// the rest is exact).
__device__ __forceinline__ void split_f32(const vec16& lo, const vec16& hi, vec16* parts) {
  uint32_t cut[3][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float rest = __uint_as_float(i < 4 ? lo[i & 3] : hi[i & 3]);
#pragma unroll
    for (int p = 0; p < 3; ++p) {
      cut[p][i] = __float_as_uint(rest) & 0xffff0000u;
      rest -= __uint_as_float(cut[p][i]);
    }
  }
#pragma unroll
  for (int p = 0; p < 3; ++p)
#pragma unroll
    for (int j = 0; j < 4; ++j) parts[p][j] = __builtin_amdgcn_perm(cut[p][j + 4], cut[p][j], 0x07060302u);
}

// Which rows of y, and whose matrix, slot number `slot` of tiles of `cols` rows
// covers.  Every expert's rows make ceil(n / cols) tiles, in order; the dropped
// rows behind them make tiles of a matrix number `experts`, to be filled with
// zeros.  Found by every wave for itself: 64 experts at once.  false: no tile.
__device__ __forceinline__ bool find_tile(const Q4Args& a, uint32_t slot, uint32_t cols, int* expert, uint32_t* first,
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

template <int DT>
__device__ __forceinline__ void store_y(const Q4Args& a, uint32_t n, int64_t m, float v) {
  typedef Type<DT> T;
  char* p = a.y + n * a.ldy;
  if (DT == 0 || a.y_f32)
    reinterpret_cast<float*>(p)[m] = v;
  else
    reinterpret_cast<typename T::elt*>(p)[m] = T::narrow(v);
}

__device__ __forceinline__ float silu(float v) { return v / (1.f + __expf(-v)); }

}  // namespace ebag
