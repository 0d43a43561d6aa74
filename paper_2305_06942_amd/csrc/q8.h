// What the kernels with 8-bit weights share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"
#include "products.h"
#include "vec16.h"

namespace ebag {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x16 __attribute__((ext_vector_type(16)));

// Bytes of a row of codes: whole cache lines, so that rows begin on one and every
// step of a product is whole.  Rows of x end in zeros, so what stands behind a
// row of weights does not matter.
constexpr int64_t kQ8Line = 128;
constexpr int64_t q8_pitch(int64_t K) { return (K + kQ8Line - 1) / kQ8Line * kQ8Line; }

struct Q8Args {
  const int8_t* codes;
  const float* scales;
  const int8_t* xq;         // rows of x in 8 bits
  const float* xs;          // and their scales
  char* y;
  const int32_t* offsets;   // nullptr: one matrix, all rows
  const int32_t* src;       // nullptr: row p of x
  int64_t ldy;              // bytes
  int64_t pitch;
  int64_t M;                // rows of a matrix
  int64_t out_rows;         // of those, the ones a column of y belongs to: M, or M / 2 with glu
  int64_t x_rows;
  uint32_t rows;            // of y
  int32_t experts;
  int32_t glu;
  int32_t y_type;
  Divisor by_choices;
  Divisor by_tiles;         // workgroups that share the rows of x, each with its rows of weights
  // The matrix-product kernel.
  uint32_t whole;           // workgroups in whole rounds of all XCDs
};

// Row of x that belongs to row n of y.
__device__ __forceinline__ int64_t q8_x_row(const Q8Args& a, uint32_t n) {
  const int64_t row = a.src ? (int64_t)divide_by(a.by_choices, (uint32_t)a.src[n] & 0x7fffffffu) : (int64_t)n;
  return row < a.x_rows ? row : a.x_rows - 1;
}

__device__ __forceinline__ void q8_store(const Q8Args& a, uint32_t n, int64_t m, float v) {
  char* p = a.y + n * a.ldy;
  if (a.y_type == EBAG_F32)
    reinterpret_cast<float*>(p)[m] = v;
  else if (a.y_type == EBAG_F16)
    reinterpret_cast<_Float16*>(p)[m] = Type<1>::narrow(v);
  else
    reinterpret_cast<__bf16*>(p)[m] = Type<2>::narrow(v);
}

// Rows of weights and rows of x of a workgroup of the matrix-product kernel.
enum Q8Tile { Q8_256x64, Q8_512x128, Q8_256x256 };
constexpr int q8_tile_w(Q8Tile t) { return t == Q8_512x128 ? 512 : 256; }
constexpr int q8_tile_x(Q8Tile t) { return t == Q8_256x64 ? 64 : t == Q8_512x128 ? 128 : 256; }

// tiles: of 16 rows of weights of a wave; x_tiles: of 16 rows of x; waves: of four, that have different rows of weights.
void launch_q8_few(const Q8Args& a, int tiles, int x_tiles, int waves, unsigned grid, hipStream_t stream);
void launch_q8_tile(const Q8Args& a, Q8Tile kind, unsigned grid, hipStream_t stream);

}  // namespace ebag
