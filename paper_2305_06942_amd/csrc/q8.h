// What the kernels with 8-bit weights share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"
#include "lanes.h"
#include "products.h"
#include "q8_choose.h"
#include "vec16.h"

namespace ebag {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x16 __attribute__((ext_vector_type(16)));

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
  const char* x;            // a row to be rounded by the product itself (launch_q8_own alone)
  int32_t x_type;
  int32_t K;
  Divisor by_choices;
  Divisor by_tiles;         // workgroups that share the rows of x, each with its rows of weights: of the kernel for few
                            // rows those of an XCD, or all
  int32_t spread;           // of the kernel for few rows: 3, neighbouring tiles on the eight XCDs, or 0, no order
  uint32_t tiles;           // the kernel for few rows: all of them
  Divisor by_group;         // and slots that have their turn with a workgroup's weights one after the other
  // The matrix-product kernel.
  uint32_t whole;           // workgroups in whole rounds of all XCDs
};

// Row of x that belongs to row n of y.
__device__ __forceinline__ int64_t q8_x_row(const Q8Args& a, uint32_t n) {
  const int64_t row = a.src ? (int64_t)divide_by(a.by_choices, (uint32_t)a.src[n] & 0x7fffffffu) : (int64_t)n;
  return row < a.x_rows ? row : a.x_rows - 1;
}

// A result in fp32.  Left to itself the compiler rounds some products to fp16 at once and some over fp32, and a row's results
// would differ in their last bit from kernel to kernel.
__device__ __forceinline__ float q8_result(float v) {
  asm("" : "+v"(v));
  return v;
}

__device__ __forceinline__ void q8_store(const Q8Args& a, uint32_t n, int64_t m, float v) {
  char* p = a.y + n * a.ldy;
  if (a.y_type == EBAG_F32)
    reinterpret_cast<float*>(p)[m] = v;
  else if (a.y_type == EBAG_F16)
    reinterpret_cast<_Float16*>(p)[m] = Type<1>::narrow(q8_result(v));
  else
    reinterpret_cast<__bf16*>(p)[m] = Type<2>::narrow(v);
}

// The largest over the 64 lanes, in each of them; of numbers without a sign, as whole numbers keep the order of
// floats and put NaN above infinity.
__device__ __forceinline__ uint32_t q8_larger(uint32_t a, uint32_t b) { return a > b ? a : b; }
template <int CTRL>
__device__ __forceinline__ uint32_t q8_larger_dpp(uint32_t v) {
  return q8_larger(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ uint32_t q8_largest(uint32_t v) {
  v = q8_larger_dpp<0xB1>(v);
  v = q8_larger_dpp<0x4E>(v);
  v = q8_larger_dpp<0x141>(v);
  v = q8_larger_dpp<0x140>(v);
  const u32x2 s = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = q8_larger(s[0], s[1]);
  const u32x2 t = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return q8_larger(t[0], t[1]);
}

// Eight neighbouring elements in fp32, zeros behind the row's end.
template <int DT>
__device__ __forceinline__ void q8_load8(const char* row, int at, int K, float* f) {
  typedef Type<DT> T;
  typedef typename T::elt elt;
  if (at + 8 <= K) {
#pragma unroll
    for (int v = 0; v < 8 / T::N; ++v) T::widen(load16(row + (int64_t)at * sizeof(elt) + 16 * v), f + v * T::N);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = at + i < K ? T::widen(reinterpret_cast<const elt*>(row)[at + i]) : 0.f;
  }
}

__device__ __forceinline__ float q8_scale(uint32_t top) {  // of a row whose largest size has these bits
  return top >= 0x7f800000u ? __builtin_nanf("") : __uint_as_float(top) / 127.f;
}

// The whole number nearest to x / scale, halves to even: what the product with the reciprocal gives is at most one
// off, and x less that many scales, exact up to its sign and its order with scale / 2, says which way.
struct Q8Rounder {
  float scale, inv, half, near, factor;
  bool any;
  __device__ __forceinline__ Q8Rounder(float s) {
    // Scales so small that their reciprocal would not be a number, or their half not exact, are taken 2^64 times.
    factor = s < 0x1p-60f ? 0x1p64f : 1.f;
    scale = s * factor;
    any = s > 0.f;  // not NaN
    inv = any ? 1.f / scale : 0.f;
    half = 0.5f * scale;
    near = any && factor == 1.f ? half * (1.f - 0x1p-12f) : 0.f;
  }
  __device__ __forceinline__ int code(float x) const {
    x *= factor;
    float q = rintf(x * inv);
    const float left = fmaf(-q, scale, x), size = fabsf(left);
    if (size > half || (size == half && ((int)q & 1))) q += left > 0.f ? 1.f : -1.f;
    return any ? (int)fminf(fmaxf(q, -127.f), 127.f) : 0;
  }
};

// Eight elements to codes.  Where none of them is next to the middle of two codes, the nearest number to the product with
// the reciprocal is right as it is; it stands in the low bits of its sum with 1.5 * 2^23 (5 instructions an element
// instead of 20; 8192 rows of 8192 bf16 50 -> 46 us).
__device__ __forceinline__ void q8_store8(int8_t* to, const Q8Rounder& r, const float* f) {
  constexpr float kShift = 12582912.f;
  uint32_t bits[8], w[2] = {0, 0};
  float worst = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float t = fmaf(f[i], r.inv, kShift);
    worst = fmaxf(worst, fabsf(fmaf(-(t - kShift), r.scale, f[i])));
    bits[i] = __float_as_uint(t);
  }
  if (worst < r.near) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t lo = __builtin_amdgcn_perm(bits[4 * i + 1], bits[4 * i], 0x0c0c0400u);
      const uint32_t hi = __builtin_amdgcn_perm(bits[4 * i + 3], bits[4 * i + 2], 0x04000c0cu);
      w[i] = lo | hi;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i / 4] |= ((uint32_t)r.code(f[i]) & 0xffu) << (8 * (i % 4));
  }
  *reinterpret_cast<uint2*>(to) = uint2{w[0], w[1]};
}

// silu(v), for a 16-bit y with the short reciprocal besides the short exponential: off by (|v| + 8) 2^-22 all the same.  The
// division's ten instructions are a third of the matrix-product kernel's work behind its sums.  With h = exp(v / 2) silu is
// v h / (1 + h^2) h: no step leaves the normal numbers before the result does, where exp(-v) and the reciprocal of a
// sum above 2^126 would (0 below v = -87.3, where bf16 has 2e-37 at -89 still; without that 32768 rows on 64 experts of 4096 x 2048
// took 400 us, like this 404).  Above 20 the factor of v is 1 to 2e-9.
template <bool Y32>
__device__ __forceinline__ float q8_silu(float v) {
  if (Y32) return silu<true>(v);
  const float h = __builtin_amdgcn_exp2f(0.72134752f * __builtin_fminf(v, 20.f));  // 1 / (2 ln 2)
  return v * (h * __builtin_amdgcn_rcpf(__builtin_fmaf(h, h, 1.f))) * h;
}

// tiles: of 16 rows of weights of a wave; x_tiles: of 16 rows of x; waves: of four, that have different rows of weights.
void launch_q8_few(const Q8Args& a, int tiles, int x_tiles, int waves, unsigned grid, hipStream_t stream);
// The same for a row of x of any type, of whole 16-byte vectors on 16-byte boundaries.
bool q8_own_fits(const Q8Args& a);
void launch_q8_own(const Q8Args& a, int tiles, int waves, unsigned grid, hipStream_t stream);
void launch_q8_tile(const Q8Args& a, Q8Tile kind, unsigned grid, hipStream_t stream);

}  // namespace ebag
