// Products with 8-bit weights for few rows of x: the kernel that streams the weights.
#include <hip/hip_runtime.h>

#include "gemv_ar.h"
#include "q8.h"

namespace ebag {
namespace {

// A wave has RT tiles of 16 rows of weights (with glu a tile of gate rows and the up rows
// that go with them) and NT tiles of 16 rows of x, and of their columns the part that is
// its of `split` waves.  Weights and x come straight from memory into the operands'
// registers, two lines of each row at a time and the next two on their way; sums are
// whole numbers, so the order in which the waves' parts are joined does not matter.
template <int RT, int NT>
__global__ __launch_bounds__(512) void q8_few_kernel(const Q8Args a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  constexpr int P = 2;  // lines at a time
  const int lane = threadIdx.x & 63, r16 = lane & 15, quarter = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int waves = blockDim.x >> 6, split = a.split, part = wave & (split - 1), own = wave / split;
  const uint32_t slot = divide_by(a.by_tiles, blockIdx.x), tile = blockIdx.x - slot * a.by_tiles.d;
  int expert;
  uint32_t first, end;
  if (!find_tile(a, slot, 16 * NT, &expert, &first, &end)) return;
  const int pair = a.glu ? 2 : 1;
  const int64_t wg_cols = 16 * RT / pair * (waves / split);
  const int64_t m0 = tile * wg_cols + own * (16 * RT / pair);
  if (expert == a.experts) {
    for (uint32_t i = threadIdx.x; i < 16u * NT * (uint32_t)wg_cols; i += blockDim.x) {
      const uint32_t n = first + i / (uint32_t)wg_cols;
      const int64_t m = tile * wg_cols + i % (uint32_t)wg_cols;
      if (n < end && m < a.out_rows) q8_store(a, n, m, 0.f);
    }
    return;
  }
  const int8_t* w[RT];
  const int8_t* x[NT];
#pragma unroll
  for (int b = 0; b < RT; ++b) {
    int64_t m = m0 + (pair == 2 ? 0 : 16 * b) + r16;
    m = m < a.out_rows ? m : a.out_rows - 1;
    w[b] = a.codes + ((int64_t)expert * a.M + (pair == 2 && b ? a.out_rows : 0) + m) * a.pitch + quarter * 16;
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    uint32_t n = first + 16 * t + r16;
    n = n < end ? n : end - 1;
    x[t] = a.xq + q8_x_row(a, n) * a.pitch + quarter * 16;
  }
  const int lines = (int)(a.pitch / kQ8Line);
  const int from = lines * part / split, to = lines * (part + 1) / split;
  struct Lines {
    i32x4 w[RT][2 * P], x[NT][2 * P];
  };
  auto load = [&](Lines& l, int line) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int64_t at = (int64_t)(line + p < to ? line + p : to - 1) * kQ8Line;  // a line again where there is none
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int b = 0; b < RT; ++b) l.w[b][2 * p + h] = __builtin_bit_cast(i32x4, load16(reinterpret_cast<const char*>(w[b] + at + 64 * h)));
#pragma unroll
        for (int t = 0; t < NT; ++t) l.x[t][2 * p + h] = __builtin_bit_cast(i32x4, load16(reinterpret_cast<const char*>(x[t] + at + 64 * h)));
      }
    }
  };
  i32x4 sum[RT][NT];
#pragma unroll
  for (int b = 0; b < RT; ++b)
#pragma unroll
    for (int t = 0; t < NT; ++t) sum[b][t] = i32x4{0, 0, 0, 0};
  if (from < to) {
    Lines now, next;
    load(now, from);
    for (int line = from; line < to; line += P) {
      if (line + P < to) load(next, line + P);
#pragma unroll
      for (int p = 0; p < P; ++p) {
        if (line + p >= to) break;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int b = 0; b < RT; ++b)
#pragma unroll
            for (int t = 0; t < NT; ++t)
              sum[b][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(now.x[t][2 * p + h], now.w[b][2 * p + h], sum[b][t], 0, 0, 0);
      }
      now = next;
    }
  }
  // A lane has weight row r16 and rows 4 quarter .. of x.  The first of a tile's waves finishes what all have.
  i32x4* joined = reinterpret_cast<i32x4*>(lds);
  if (split > 1) {
    if (part) {
#pragma unroll
      for (int b = 0; b < RT; ++b)
#pragma unroll
        for (int t = 0; t < NT; ++t) joined[((wave * RT + b) * NT + t) * 64 + lane] = sum[b][t];
    }
    __syncthreads();
    if (part) return;
    for (int p = 1; p < split; ++p)
#pragma unroll
      for (int b = 0; b < RT; ++b)
#pragma unroll
        for (int t = 0; t < NT; ++t) sum[b][t] += joined[(((wave + p) * RT + b) * NT + t) * 64 + lane];
  }
  const float* scales = a.scales + (int64_t)expert * a.M;
#pragma unroll
  for (int b = 0; b < RT; ++b) {
    if (pair == 2 && b) continue;
    const int64_t m = m0 + 16 * b + r16;
    if (m >= a.out_rows) continue;
    const float ws = scales[m], wu = pair == 2 ? scales[a.out_rows + m] : 0.f;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t n = first + 16 * t + 4 * quarter + i;
        if (n >= end) continue;
        const float xs = a.xs[q8_x_row(a, n)];
        float v = (float)sum[b][t][i] * (xs * ws);
        if (RT > 1 && pair == 2) {
          const float up = (float)sum[RT > 1 ? 1 : 0][t][i] * (xs * wu);
          v = (a.y_type == EBAG_F32 ? silu<true>(v) : silu<false>(v)) * up;
        }
        q8_store(a, n, m, v);
      }
  }
}

template <int RT>
void (*pick(int x_tiles))(const Q8Args) {
  return x_tiles == 1 ? q8_few_kernel<RT, 1> : x_tiles == 2 ? q8_few_kernel<RT, 2> : q8_few_kernel<RT, 4>;
}

}  // namespace

void launch_q8_few(const Q8Args& a, int tiles, int x_tiles, unsigned grid, int threads, hipStream_t stream) {
  const size_t lds = a.split > 1 ? (size_t)threads * tiles * x_tiles * 16 : 0;
  hipLaunchKernelGGL(tiles == 1 ? pick<1>(x_tiles) : pick<2>(x_tiles), dim3(grid), dim3(threads), lds, stream, a);
}

}  // namespace ebag
