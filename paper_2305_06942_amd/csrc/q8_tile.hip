// Products with 8-bit weights for many rows of x: the matrix-product kernel.
#include <hip/hip_runtime.h>

#include "gemv_ar.h"
#include "q8.h"

namespace ebag {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;
constexpr int kB = 2;           // a wave's tiles of 32 weight rows
constexpr int kStep = kQ8Line;  // columns of a step

// A workgroup has 256 rows of weights and BN rows of x, each of eight waves 64 of the
// weight rows and half of the rows of x.  Both go through LDS, two steps of 128 columns in
// turn, 16-byte pieces of a row exchanged by its number so that the lanes of an operand
// find theirs on different banks.
template <int BN>
__global__ __launch_bounds__(kThreads) void q8_tile_kernel(const Q8Args a) {
  constexpr int NT = BN / 64;                            // a wave's tiles of 32 rows of x
  constexpr int ROWS = kQ8TileRows + BN;                 // of LDS
  constexpr int STAGED = ROWS * kStep / 16 / kThreads;   // pieces of a thread
  constexpr int W_STAGED = kQ8TileRows * kStep / 16 / kThreads;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, r32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wave_m = wave & 3, wave_n = wave >> 2;
  // 32 neighbouring tiles to each XCD, whose L2 then has what they share.
  uint32_t block = blockIdx.x;
  if (block < a.whole) block = (block >> 8 << 8) + ((block & 7) << 5) + (block >> 3 & 31);
  const uint32_t quad = divide_by(a.by_tiles, block >> 2), tile = (block >> 2) - quad * a.by_tiles.d;
  const uint32_t slot = quad * 4 + (block & 3);
  int expert;
  uint32_t first, end;
  if (!find_tile(a, slot, BN, &expert, &first, &end)) return;
  const int pair = a.glu ? 2 : 1;
  const int64_t wg_m0 = (int64_t)tile * (kQ8TileRows / pair);
  if (expert == a.experts) {
    const uint32_t cols = kQ8TileRows / pair;
    for (uint32_t i = tid; i < BN * cols; i += kThreads) {
      const uint32_t n = first + i / cols;
      const int64_t m = wg_m0 + i % cols;
      if (n < end && m < a.out_rows) q8_store(a, n, m, 0.f);
    }
    return;
  }
  // Staging: a thread has piece `chunk` of rows row, row + 64, ... of weights, then of x.
  const int row0 = tid >> 3, chunk = tid & 7;
  const int8_t* from[STAGED];
#pragma unroll
  for (int i = 0; i < STAGED; ++i) {
    if (i < W_STAGED) {
      const int r = row0 + 64 * i;
      int64_t m = wg_m0 + (pair == 2 ? r / 64 * 32 + r % 32 : r);
      m = m < a.out_rows ? m : a.out_rows - 1;
      if (pair == 2 && r / 32 % 2) m += a.out_rows;
      from[i] = a.codes + ((int64_t)expert * a.M + m) * a.pitch + chunk * 16;
    } else {
      uint32_t n = first + row0 + 64 * (i - W_STAGED);
      n = n < end ? n : end - 1;
      from[i] = a.xq + q8_x_row(a, n) * a.pitch + chunk * 16;
    }
  }
  char* to = lds + row0 * kStep + (chunk ^ (row0 & 7)) * 16;  // rows 64 apart have the same exchange
  constexpr int BUFFER = ROWS * kStep;
  const char* w_at = lds + (wave_m * 64 + r32) * kStep;
  const char* x_at = lds + (kQ8TileRows + wave_n * (BN / 2) + r32) * kStep;
  const int turn = r32 & 7;

  i32x16 sum[kB][NT];
#pragma unroll
  for (int b = 0; b < kB; ++b)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) sum[b][t][i] = 0;

  vec16 staged[STAGED];
  auto load = [&](int step) {
#pragma unroll
    for (int i = 0; i < STAGED; ++i) staged[i] = load16(reinterpret_cast<const char*>(from[i]) + (int64_t)step * kStep);
  };
  auto store = [&](int buffer) {
#pragma unroll
    for (int i = 0; i < STAGED; ++i) *reinterpret_cast<vec16*>(to + buffer * BUFFER + i * 64 * kStep) = staged[i];
  };
  auto multiply = [&](int buffer, int slice) {
    const int piece = ((slice * 2 + half) ^ turn) * 16 + buffer * BUFFER;
    i32x4 x[NT], w[kB];
#pragma unroll
    for (int t = 0; t < NT; ++t) x[t] = *reinterpret_cast<const i32x4*>(x_at + 32 * t * kStep + piece);
#pragma unroll
    for (int b = 0; b < kB; ++b) w[b] = *reinterpret_cast<const i32x4*>(w_at + 32 * b * kStep + piece);
#pragma unroll
    for (int b = 0; b < kB; ++b)
#pragma unroll
      for (int t = 0; t < NT; ++t) sum[b][t] = __builtin_amdgcn_mfma_i32_32x32x32_i8(x[t], w[b], sum[b][t], 0, 0, 0);
  };
  const int steps = (int)(a.pitch / kStep);
  load(0);
  store(0);
  if (steps > 1) load(1);
  __syncthreads();
  for (int step = 0; step < steps; ++step) {
    const int buffer = step & 1;
    multiply(buffer, 0);
    multiply(buffer, 1);
    if (step + 1 < steps) store(buffer ^ 1);
    if (step + 2 < steps) load(step + 2);
    multiply(buffer, 2);
    multiply(buffer, 3);
    __syncthreads();
  }
  // A lane has weight row r32 and, in element i, row 8 (i / 4) + 4 half + i % 4 of x.
  const float* scales = a.scales + (int64_t)expert * a.M;
#pragma unroll
  for (int b = 0; b < kB; ++b) {
    if (pair == 2 && b) continue;
    const int64_t m = wg_m0 + (pair == 2 ? wave_m * 32 : wave_m * 64 + 32 * b) + r32;
    if (m >= a.out_rows) continue;
    const float ws = scales[m], wu = pair == 2 ? scales[a.out_rows + m] : 0.f;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const uint32_t n = first + wave_n * (BN / 2) + 32 * t + 8 * (i / 4) + 4 * half + i % 4;
        if (n >= end) continue;
        const float xs = a.xs[q8_x_row(a, n)];
        float v = (float)sum[b][t][i] * (xs * ws);
        if (pair == 2) {
          const float up = (float)sum[1][t][i] * (xs * wu);
          v = (a.y_type == EBAG_F32 ? silu<true>(v) : silu<false>(v)) * up;
        }
        q8_store(a, n, m, v);
      }
  }
}

}  // namespace

void launch_q8_tile(const Q8Args& a, int x_rows, unsigned grid, hipStream_t stream) {
  const size_t lds = 2 * (size_t)(kQ8TileRows + x_rows) * kStep;
  hipLaunchKernelGGL(x_rows == 256 ? q8_tile_kernel<256> : x_rows == 128 ? q8_tile_kernel<128> : q8_tile_kernel<64>, dim3(grid),
                     dim3(kThreads), lds, stream, a);
}

}  // namespace ebag
