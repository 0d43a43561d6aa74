// Products with 8-bit weights for many rows of x: the matrix-product kernel.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "gemv_ar.h"
#include "q8.h"

namespace ebag {
namespace {

constexpr int kThreads = 256;
constexpr int kStep = kQ8Line;  // columns of a step
constexpr int kSlices = kStep / 32;

// WW x WX waves, four in all, have 32 TW rows of weights and 32 TX rows of x each.  Both go
// through LDS, two steps of 128 columns in turn, 16-byte pieces of a row exchanged by
// its number so that the lanes of an operand find theirs on different banks.
template <int WW, int WX, int TW, int TX, bool GLU, int ELT>
__global__ __launch_bounds__(kThreads, 1) void q8_tile_kernel(const Q8Args a) {
  constexpr int BW = 32 * TW * WW, BX = 32 * TX * WX, ROWS = BW + BX;
  constexpr int W_STAGED = BW / 32, STAGED = ROWS / 32;  // pieces of a thread, 32 rows apart
  constexpr int BUFFER = ROWS * kStep;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, r32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wave_w = wave % WW, wave_x = wave / WW;
  // 32 neighbouring tiles to each XCD, whose L2 then has what they share.
  uint32_t block = blockIdx.x;
  if (block < a.whole) block = (block >> 8 << 8) + ((block & 7) << 5) + (block >> 3 & 31);
  const uint32_t quad = divide_by(a.by_tiles, block >> 2), tile = (block >> 2) - quad * a.by_tiles.d;
  const uint32_t slot = quad * 4 + (block & 3);
  int expert;
  uint32_t first, end;
  if (!find_tile(a, slot, BX, &expert, &first, &end)) return;
  expert = __builtin_amdgcn_readfirstlane(expert);
  constexpr int pair = GLU ? 2 : 1;
  const int64_t wg_m0 = (int64_t)tile * (BW / pair);
  if (expert == a.experts) {
    const uint32_t cols = BW / pair;
    for (uint32_t i = tid; i < BX * cols; i += kThreads) {
      const uint32_t n = first + i / cols;
      const int64_t m = wg_m0 + i % cols;
      if (n < end && m < a.out_rows) q8_store(a, n, m, 0.f);
    }
    return;
  }
  // Staging: a thread has piece `chunk` of rows row0, row0 + 32, ... of weights, then of x.  With glu every second 32
  // rows are up rows, those of the gate rows before them.
  const int row0 = tid >> 3, chunk = tid & 7;
  const int64_t w_row = wg_m0 < a.out_rows ? wg_m0 : a.out_rows - 1;
  const int8_t* w_from = a.codes + ((int64_t)expert * a.M + w_row) * a.pitch;
  uint32_t w_at[W_STAGED];
  const int8_t* x_from[STAGED - W_STAGED];
#pragma unroll
  for (int i = 0; i < W_STAGED; ++i) {
    int64_t m = wg_m0 + (pair == 2 ? i / 2 * 32 : i * 32) + row0;
    m = (m < a.out_rows ? m : a.out_rows - 1) - w_row;
    w_at[i] = (uint32_t)m * (uint32_t)a.pitch + chunk * 16;
  }
  const int64_t up = pair == 2 ? a.out_rows * a.pitch : 0;
#pragma unroll
  for (int i = 0; i < STAGED - W_STAGED; ++i) {
    uint32_t n = first + row0 + 32 * i;
    n = n < end ? n : end - 1;
    x_from[i] = a.xq + q8_x_row(a, n) * a.pitch + chunk * 16;
  }
  char* to = lds + row0 * kStep + (chunk ^ (row0 >> 1 & 7)) * 16;  // rows 32 apart have the same exchange
  const char* w_lds = lds + (wave_w * (32 * TW) + r32) * kStep;
  const char* x_lds = lds + (BW + wave_x * (32 * TX) + r32) * kStep;
  const int turn = r32 >> 1 & 7;

  i32x16 sum[TW][TX];
#pragma unroll
  for (int b = 0; b < TW; ++b)
#pragma unroll
    for (int t = 0; t < TX; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) sum[b][t][i] = 0;

  vec16 staged[STAGED];
  struct Operands {
    i32x4 w[TW], x[TX];
  };
  Operands even, odd;
  auto load = [&](int i, int step) {
    const int64_t at = (int64_t)step * kStep;
    staged[i] = load16(i < W_STAGED ? reinterpret_cast<const char*>(w_from + (i & 1 ? up : 0) + at) + w_at[i < W_STAGED ? i : 0]
                                    : reinterpret_cast<const char*>(x_from[i < W_STAGED ? 0 : i - W_STAGED] + at));
  };
  auto store = [&](int i, int buffer) { *reinterpret_cast<vec16*>(to + buffer * BUFFER + i * 32 * kStep) = staged[i]; };
  // Operand number i, in the order in which the products need them.
  auto fetch = [&](Operands& o, int buffer, int slice, int i) {
    const int piece = ((slice * 2 + half) ^ turn) * 16 + buffer * BUFFER;
    if (i > 0 && i <= TW)
      o.w[i > 0 && i <= TW ? i - 1 : 0] = *reinterpret_cast<const i32x4*>(w_lds + 32 * (i - 1) * kStep + piece);
    else
      o.x[i ? i - TW : 0] = *reinterpret_cast<const i32x4*>(x_lds + 32 * (i ? i - TW : 0) * kStep + piece);
  };
  // A slice's products, with other work between them: kept where it stands, so that a wave alone on its SIMD always
  // has products under way while it waits for memory.
  constexpr int GROUPS = TW + TX, EACH = TW * TX / GROUPS;
  static_assert(EACH * GROUPS == TW * TX, "");
  auto multiply = [&](const Operands& o, auto other) __attribute__((always_inline)) {
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
#pragma unroll
      for (int i = g * EACH; i < (g + 1) * EACH; ++i)
        sum[i % TW][i / TW] = __builtin_amdgcn_mfma_i32_32x32x32_i8(o.w[i % TW], o.x[i / TW], sum[i % TW][i / TW], 0, 0, 0);
      other(g);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // One step's products.  Its first operands are in registers; the next step's rows, loaded a step ago, go to the
  // other buffer, which nobody reads any more, while the second and third slices are multiplied, and the loads of the
  // step after that take their registers.  After the third slice every wave has read what it needs of this buffer and
  // stored its part of the other: one barrier a step, with a slice's products to follow at once.
  auto work = [&](int buffer, int step, auto stores, auto loads) __attribute__((always_inline)) {
    constexpr bool STORES = decltype(stores)::value, LOADS = decltype(loads)::value;
    auto move = [&](int part, int g) __attribute__((always_inline)) {  // the pieces between whose products this group is
      constexpr int MOVES = 2 * GROUPS;
      const int from = (part * GROUPS + g) * STAGED / MOVES, to = (part * GROUPS + g + 1) * STAGED / MOVES;
#pragma unroll
      for (int i = from; i < to; ++i) {
        if (STORES) store(i, buffer ^ 1);
        if (LOADS) load(i, step + 2);
      }
    };
    multiply(even, [&](int g) __attribute__((always_inline)) { fetch(odd, buffer, 1, g); });
    multiply(odd, [&](int g) __attribute__((always_inline)) {
      fetch(even, buffer, 2, g);
      move(0, g);
    });
    multiply(even, [&](int g) __attribute__((always_inline)) {
      fetch(odd, buffer, 3, g);
      move(1, g);
    });
    __syncthreads();
    multiply(odd, [&](int g) __attribute__((always_inline)) {
      if (STORES) fetch(even, buffer ^ 1, 0, g);
    });
  };
  const int steps = (int)(a.pitch / kStep);
#pragma unroll
  for (int i = 0; i < STAGED; ++i) load(i, 0);
#pragma unroll
  for (int i = 0; i < STAGED; ++i) store(i, 0);
  if (steps > 1) {
#pragma unroll
    for (int i = 0; i < STAGED; ++i) {
      load(i, 1);
      __builtin_amdgcn_sched_barrier(0);  // in the order in which they are waited for
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) fetch(even, 0, 0, i);
  int step = 0;
  for (; step + 2 < steps; ++step) work(step & 1, step, std::true_type(), std::true_type());
  if (step + 1 < steps) {
    work(step & 1, step, std::true_type(), std::false_type());
    ++step;
  }
  work(step & 1, step, std::false_type(), std::false_type());

  // A lane has row r32 of x and, in element i, weight row 8 (i / 4) + 4 half + i % 4: four neighbours, which go to LDS
  // as one piece, 32 rows of x at a time, and from there to y in whole rows.
  constexpr int COLS = 32 * TW / pair, PITCH = COLS * ELT + 16;  // columns of y that the wave has; bytes of a row in LDS
  constexpr int VEC = 16 / ELT, PER_ROW = COLS / VEC;            // elements of a vector, vectors of a row
  const int64_t m0 = wg_m0 + wave_w * COLS;
  const int64_t left = a.out_rows - m0;                          // columns of y from the wave's first on
  const float* scales = a.scales + (int64_t)expert * a.M;
  float ws[TW][16], xs[TX];
#pragma unroll
  for (int b = 0; b < TW; ++b)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int col = (GLU ? b / 2 : b) * 32 + 8 * q + 4 * half;
      const float* from = scales + (GLU && b % 2 ? a.out_rows : 0);
      if (col + 4 <= left) {
        Type<0>::widen(load16(reinterpret_cast<const char*>(from + m0 + col)), &ws[b][4 * q]);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) ws[b][4 * q + i] = from[col + i < left ? m0 + col + i : a.out_rows - 1];
      }
    }
#pragma unroll
  for (int t = 0; t < TX; ++t) {
    const uint32_t n = first + wave_x * (32 * TX) + 32 * t + r32;
    xs[t] = a.xs[q8_x_row(a, n < end ? n : end - 1)];
  }
  __syncthreads();
  char* mine = lds + wave * (32 * PITCH);
#pragma unroll
  for (int t = 0; t < TX; ++t) {
    const uint32_t n0 = first + wave_x * (32 * TX) + 32 * t;
    if (n0 >= end) break;
#pragma unroll
    for (int b = 0; b < TW; b += pair)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float v[8] = {};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int at = 4 * q + i;
          v[i] = (float)sum[b][t][at] * (xs[t] * ws[b][at]);
          if (GLU) v[i] = silu<ELT == 4>(v[i]) * ((float)sum[b + pair - 1][t][at] * (xs[t] * ws[b + pair - 1][at]));
        }
        char* to = mine + r32 * PITCH + (b / pair * 32 + 8 * q + 4 * half) * ELT;
        if constexpr (ELT == 4) {
          *reinterpret_cast<vec16*>(to) = Type<0>::narrow(v);
        } else {
          const vec16 p = a.y_type == EBAG_F16 ? Type<1>::narrow(v) : Type<2>::narrow(v);
          *reinterpret_cast<uint2*>(to) = uint2{p[0], p[1]};
        }
      }
    __builtin_amdgcn_wave_barrier();
    constexpr int LANES = PER_ROW < 64 ? PER_ROW : 64;  // of a row
    const int r0 = lane / LANES, c = lane % LANES * VEC;
    char* out = a.y + (int64_t)(n0 + r0) * a.ldy + (m0 + c) * ELT;
    const char* at = mine + r0 * PITCH + c * ELT;
    if (c < left) {
#pragma unroll
      for (int i = 0; i < LANES / 2; ++i) {
        if (n0 + r0 + i * (64 / LANES) >= end) break;
        char* row = out + (int64_t)i * (64 / LANES) * a.ldy;
        const vec16 v = *reinterpret_cast<const vec16*>(at + i * (64 / LANES) * PITCH);
        if (c + VEC <= left) {
          store16(row, v);
        } else {
#pragma unroll
          for (int e = 0; e < VEC; ++e)
            if (c + e < left) {
              if constexpr (ELT == 4)
                reinterpret_cast<uint32_t*>(row)[e] = v[e];
              else
                reinterpret_cast<uint16_t*>(row)[e] = (uint16_t)(e & 1 ? v[e / 2] >> 16 : v[e / 2] & 0xffffu);
            }
        }
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

template <int WW, int WX, int TW, int TX>
void launch(const Q8Args& a, unsigned grid, hipStream_t stream) {
  constexpr size_t stages = 2 * (size_t)(32 * TW * WW + 32 * TX * WX) * kStep, out = 4 * 32 * (32 * TW * 4 + 16);
  const bool f32 = a.y_type == EBAG_F32;
  hipLaunchKernelGGL((a.glu ? f32 ? q8_tile_kernel<WW, WX, TW, TX, true, 4> : q8_tile_kernel<WW, WX, TW, TX, true, 2>
                      : f32 ? q8_tile_kernel<WW, WX, TW, TX, false, 4>
                            : q8_tile_kernel<WW, WX, TW, TX, false, 2>),
                     dim3(grid), dim3(kThreads), stages > out ? stages : out, stream, a);
}

}  // namespace

void launch_q8_tile(const Q8Args& a, Q8Tile kind, unsigned grid, hipStream_t stream) {
  switch (kind) {
    case Q8_256x256: return launch<2, 2, 4, 4>(a, grid, stream);
    case Q8_512x128: return launch<4, 1, 4, 4>(a, grid, stream);
    default: return launch<4, 1, 2, 2>(a, grid, stream);
  }
}

}  // namespace ebag
