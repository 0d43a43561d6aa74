// Products with 8-bit weights for many rows of x: the matrix-product kernel.
//
// y[n][m] = xs[n] scales[m] sum_k xq[n][k] codes[m][k], the sums exact in 32 bits.  Bound by the matrix
// instructions, and those by power: with numbers that change, 16x16x64 ones alone run at 3700 to 3900 Tops
// (4900 at 2.4 GHz with operands that never change; 32x32x32 ones 3430).  Of the about 2800 cycles
// of a step of 128 columns (256 x 256 sums) 2092 are theirs; loads from LDS add 120, stores into it 360, loads from memory
// 210, measured one by one.  Rows from memory straight into LDS were no faster (22 bytes a cycle of a CU, where the
// way through registers has 70), nor operands two steps ahead in registers (spills).  8192 x 8192 x 8192 in bf16: 410 to 420 us,
// 2620 to 2680 Tops, once the card's power control has settled; of 60 calls on a card idle before, the first four take 430 us, the next
// fall back to 560 and recover within 50 (median 434 to 450).  32768 x 4096 x 2048: 271 us, of which beginnings 30 and results 50.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "gemv_ar.h"
#include "q8.h"

namespace ebag {
namespace {

constexpr int kThreads = 256;
constexpr int kStep = kQ8Line;  // columns of a step

// Sums stay where they are.  With the compiler's builtin, whose sums may move, it moves them: 264 moves a step (8192 x
// 8192 x 8192: 778 us, like this 412).  What the compiler then does not see are the wait states between a matrix
// instruction and others on its sums: settle() keeps them, behind the first values and ahead of the results' use.
__device__ __forceinline__ void add_product(i32x4& sum, const i32x4& w, const i32x4& x) {
  asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(sum) : "v"(w), "v"(x));
}
template <int N>
__device__ __forceinline__ void settle(i32x4 (&sum)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+a"(sum[i]));
  asm volatile("s_nop 15\n\ts_nop 15");
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+a"(sum[i]));
}

// WW x WX waves, four in all, have 16 TW rows of weights and 16 TX rows of x each.  Both go
// through LDS, two steps of 128 columns in turn, 16-byte pieces of a row exchanged by
// its number so that the lanes of an operand find theirs on different banks.
template <int WW, int WX, int TW, int TX, bool GLU, int DT>
__global__ __launch_bounds__(kThreads, 1) void q8_tile_kernel(const Q8Args a) {
  constexpr int BW = 16 * TW * WW, BX = 16 * TX * WX, ROWS = BW + BX;
  constexpr int W_STAGED = BW / 32, STAGED = ROWS / 32;  // pieces of a thread, 32 rows apart
  constexpr int BUFFER = ROWS * kStep;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int tid = threadIdx.x, lane = tid & 63, quarter = lane >> 4, r16 = lane & 15;
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
  const char* w_lds = lds + (wave_w * (16 * TW) + r16) * kStep;
  const char* x_lds = lds + (BW + wave_x * (16 * TX) + r16) * kStep;
  const int turn = r16 >> 1 & 7;

  i32x4 sum[TW][TX];
#pragma unroll
  for (int b = 0; b < TW; ++b)
#pragma unroll
    for (int t = 0; t < TX; ++t) sum[b][t] = i32x4{0, 0, 0, 0};
#pragma unroll
  for (int b = 0; b < TW; ++b) settle(sum[b]);

  vec16 staged[STAGED];
  i32x4 w_now[TW], x_now[2][2];  // a slice's weights; two tiles of x, and the next two
  auto load = [&](int i, int step) {
    const int64_t at = (int64_t)step * kStep;
    staged[i] = load16(i < W_STAGED ? reinterpret_cast<const char*>(w_from + (i & 1 ? up : 0) + at) + w_at[i < W_STAGED ? i : 0]
                                    : reinterpret_cast<const char*>(x_from[i < W_STAGED ? 0 : i - W_STAGED] + at));
  };
  auto store = [&](int i, int buffer) { *reinterpret_cast<vec16*>(to + buffer * BUFFER + i * 32 * kStep) = staged[i]; };
  auto piece_of = [&](int buffer, int slice) { return ((slice * 4 + quarter) ^ turn) * 16 + buffer * BUFFER; };
  auto fetch_w = [&](int b, int piece) { w_now[b] = *reinterpret_cast<const i32x4*>(w_lds + 16 * b * kStep + piece); };
  auto fetch_x = [&](int t, int piece) {
    x_now[t / 2 & 1][t & 1] = *reinterpret_cast<const i32x4*>(x_lds + 16 * t * kStep + piece);
  };
  // A slice's products, two tiles of x at a time with each of weights in turn, and behind every two products what is to
  // be done besides: kept where it stands, so that a wave alone on its SIMD always has products under way while it
  // waits for memory.  The next two tiles of x are fetched meanwhile, and with the last two the next slice's weights,
  // into the registers of those that have no more products: both 2 TW products ahead of their use.
  constexpr int GROUPS = TX / 2 * TW;
  static_assert(TX % 4 == 0, "a slice's first tiles of x are in the first registers");
  auto multiply = [&](auto fetches, int piece, int next, auto other) __attribute__((always_inline)) {
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      const int t = g / TW * 2, b = g % TW;
      other(g);
      add_product(sum[b][t], w_now[b], x_now[t / 2 & 1][0]);
      add_product(sum[b][t + 1], w_now[b], x_now[t / 2 & 1][1]);
      const bool last = t == TX - 2;
      if (!last && b < 2) fetch_x(t + 2 + b, piece);
      if (last && decltype(fetches)::value) {
        fetch_w(b, next);
        if (b < 2) fetch_x(b, next);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // One step's products.  Its first operands are in registers; the next step's rows, loaded a step ago, go to the
  // other buffer, which nobody reads any more, and the loads of the step after that take their registers.  When the
  // last two tiles of x have their turn, every wave has what it needs of this buffer and has stored its part of the
  // other: one barrier a step, with products to follow at once.
  auto work = [&](int buffer, int step, auto stores, auto loads) __attribute__((always_inline)) {
    constexpr bool STORES = decltype(stores)::value, LOADS = decltype(loads)::value;
    constexpr int MOVES = 2 * GROUPS - TW;  // groups with room for moves
    auto move = [&](int g) __attribute__((always_inline)) {
#pragma unroll
      for (int i = g * STAGED / MOVES; i < (g + 1) * STAGED / MOVES; ++i) {
        if (STORES) store(i, buffer ^ 1);
        if (LOADS) load(i, step + 2);
      }
    };
    const int second = piece_of(buffer, 1), next = piece_of(buffer ^ 1, 0);
    multiply(std::true_type(), piece_of(buffer, 0), second, move);
    multiply(stores, second, next, [&](int g) __attribute__((always_inline)) {
      if (g < GROUPS - TW) move(GROUPS + g);
      if (STORES && g == GROUPS - TW) __syncthreads();
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
  float xs[TX];  // here already, as a row's number may have to be loaded first
#pragma unroll
  for (int t = 0; t < TX; ++t) {
    const uint32_t n = first + wave_x * (16 * TX) + 16 * t + r16;
    xs[t] = a.xs[q8_x_row(a, n < end ? n : end - 1)];
  }
  __syncthreads();
#pragma unroll
  for (int b = 0; b < TW; ++b) fetch_w(b, piece_of(0, 0));
#pragma unroll
  for (int t = 0; t < 2; ++t) fetch_x(t, piece_of(0, 0));
  int step = 0;
  for (; step + 2 < steps; ++step) work(step & 1, step, std::true_type(), std::true_type());
  if (step + 1 < steps) {
    work(step & 1, step, std::true_type(), std::false_type());
    ++step;
  }
  // A lane has row r16 of x and weight rows 4 quarter ...: four neighbours, which go to LDS as one piece, 32 rows of x at
  // a time, and from there to y in whole rows.  With glu tiles 0 and 1 of every four are of gate rows, 2 and 3 of up rows.
  // The scales are loaded ahead of the last step's products.
  constexpr int ELT = DT == 0 ? 4 : 2;
  constexpr int COLS = 16 * TW / pair, PITCH = COLS * ELT + 16;  // columns of y that the wave has; bytes of a row in LDS
  constexpr int VEC = 16 / ELT, PER_ROW = COLS / VEC;            // elements of a vector, vectors of a row
  const int64_t m0 = wg_m0 + wave_w * COLS;
  const int64_t left = a.out_rows - m0;                          // columns of y from the wave's first on
  const float* scales = a.scales + (int64_t)expert * a.M;
  auto col_of = [&](int b) { return (GLU ? b / 4 * 2 + b % 2 : b) * 16 + 4 * quarter; };
  float ws[TW][4];
#pragma unroll
  for (int b = 0; b < TW; ++b) {
    const int col = col_of(b);
    const float* from = scales + (GLU && b % 4 >= 2 ? a.out_rows : 0);
    if (col + 4 <= left) {
      Type<0>::widen(load16(reinterpret_cast<const char*>(from + m0 + col)), ws[b]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) ws[b][i] = from[col + i < left ? m0 + col + i : a.out_rows - 1];
    }
  }
  work(step & 1, step, std::false_type(), std::false_type());
#pragma unroll
  for (int b = 0; b < TW; ++b) settle(sum[b]);

  __syncthreads();
  char* mine = lds + wave * (32 * PITCH);
#pragma unroll
  for (int t0 = 0; t0 < TX; t0 += 2) {
    const uint32_t n0 = first + wave_x * (16 * TX) + 16 * t0;
    if (n0 >= end) break;
#pragma unroll
    for (int t = t0; t < t0 + 2; ++t)
#pragma unroll
      for (int b = 0; b < TW; ++b) {
        if (GLU && b % 4 >= 2) continue;
        float v[8] = {};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[i] = (float)sum[b][t][i] * (xs[t] * ws[b][i]);
          if (GLU) v[i] = q8_silu<DT == 0>(v[i]) * ((float)sum[GLU ? b + 2 : b][t][i] * (xs[t] * ws[GLU ? b + 2 : b][i]));
          if (DT == 1) v[i] = q8_result(v[i]);
        }
        char* to = mine + ((t - t0) * 16 + r16) * PITCH + col_of(b) * ELT;
        const vec16 p = Type<DT>::narrow(v);
        if constexpr (DT == 0)
          *reinterpret_cast<vec16*>(to) = p;
        else
          *reinterpret_cast<uint2*>(to) = uint2{p[0], p[1]};
      }
    __builtin_amdgcn_wave_barrier();
    constexpr int LANES = PER_ROW < 64 ? PER_ROW : 64;  // of a row
    const int r0 = lane / LANES, c = lane % LANES * VEC;
    char* out = a.y + (int64_t)(n0 + r0) * a.ldy + (m0 + c) * ELT;
    const char* at = mine + r0 * PITCH + c * ELT;
    constexpr int ROUND = 64 / LANES;  // rows at a time
    if (n0 + 32 <= end && COLS <= left) {
#pragma unroll
      for (int i = 0; i < 32 / ROUND; ++i)
        store16(out + (int64_t)(i * ROUND) * a.ldy, *reinterpret_cast<const vec16*>(at + i * ROUND * PITCH));
    } else {
      const int64_t fit = left - c;
#pragma unroll 1
      for (int i = 0; i < 32 && n0 + r0 + i < end && fit > 0; i += ROUND) {
        char* row = out + i * a.ldy;
        const char* from = at + i * PITCH;
        if (fit >= VEC) {
          store16(row, *reinterpret_cast<const vec16*>(from));
        } else {
#pragma unroll 1
          for (int e = 0; e < fit; ++e)
            reinterpret_cast<typename Type<DT>::elt*>(row)[e] = reinterpret_cast<const typename Type<DT>::elt*>(from)[e];
        }
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

template <int WW, int WX, int TW, int TX>
void launch(const Q8Args& a, unsigned grid, hipStream_t stream) {
  constexpr size_t stages = 2 * (size_t)(16 * TW * WW + 16 * TX * WX) * kStep, out = 4 * 32 * (16 * TW * 4 + 16);
  void (*fn)(const Q8Args) = a.y_type == EBAG_F32   ? a.glu ? q8_tile_kernel<WW, WX, TW, TX, true, 0> : q8_tile_kernel<WW, WX, TW, TX, false, 0>
                             : a.y_type == EBAG_F16 ? a.glu ? q8_tile_kernel<WW, WX, TW, TX, true, 1> : q8_tile_kernel<WW, WX, TW, TX, false, 1>
                             : a.glu                ? q8_tile_kernel<WW, WX, TW, TX, true, 2>
                                                    : q8_tile_kernel<WW, WX, TW, TX, false, 2>;
  hipLaunchKernelGGL(fn, dim3(grid), dim3(kThreads), stages > out ? stages : out, stream, a);
}

}  // namespace

void launch_q8_tile(const Q8Args& a, Q8Tile kind, unsigned grid, hipStream_t stream) {
  switch (kind) {
    case Q8_256x256: return launch<2, 2, 8, 8>(a, grid, stream);
    case Q8_512x128: return launch<4, 1, 8, 8>(a, grid, stream);
    default: return launch<4, 1, 4, 4>(a, grid, stream);
  }
}

}  // namespace ebag
