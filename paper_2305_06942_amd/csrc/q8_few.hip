// Products with 8-bit weights for few rows of x: the kernel that streams the weights.
//
// Bound by memory: every weight is read once (one to 128 rows of x), 5.6 to 5.8 of the 6.4 TB/s that a plain read reaches,
// where the matrix is large (16 rows x 65536 x 8192 in bf16 92 us); by the chain launch, weights, join of the
// columns' parts, store where it is small (one row x 4096 x 4096 6.5 us, of which bytes 2.6).  Weights go into LDS without
// registers, so a CU has most of a ring of up to 160 KB of them under way (64 rows x 65536 x 8192: 104 us; with loads into
// registers 198).
#include <hip/hip_runtime.h>

#include "gemv_ar.h"
#include "q8.h"

namespace ebag {
namespace {

constexpr int kCuLds = 160 * 1024;

// 16 bytes of each lane from memory into LDS, `to` and behind, without a register between: the wave may have as many
// under way as there is LDS for them.  The compiler's own builtin would have every later load from LDS wait for all of
// them; here the kernel waits itself (arrived()), by their number, as they arrive in order.  The LDS address goes in m0, as an
// operand, so that the compiler knows of it; the s_nop is the wait state behind its write.
__device__ __forceinline__ void copy_to_lds(uint32_t to, const int8_t* from) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"{m0}"(to), "v"(from) : "memory");
}
// Waits until at most N copies of this wave are under way, and for the other waves to have come as far.
template <int N>
__device__ __forceinline__ void arrived() {
  static_assert(N <= 63, "");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// Of a workgroup's WAVES waves WW have different rows of weights, RT tiles of 16 each (with glu tiles of gate rows
// and the up rows that go with them), and WK = WAVES / WW share the columns, each a part of whole lines of 128.  All of
// them have the same NT tiles of 16 rows of x.  A line of each row goes through LDS, in a ring of STAGES of them.
// Sums are whole numbers, so the order in which the parts of the columns are joined does not matter.
template <int RT, int NT, int WW, int WAVES, bool OWN>
struct Few {
  static constexpr int WK = WAVES / WW;
  static constexpr int W_ROWS = 16 * RT * WW, X_ROWS = OWN ? 0 : 16 * NT, ROWS = W_ROWS + X_ROWS;  // of a part of the columns
  static constexpr int STAGE = WK * ROWS * (int)kQ8Line;
  static constexpr int X_COPIES = X_ROWS / 8 / WW, COPIES = 2 * RT + X_COPIES;           // of a wave, eight rows each
  static_assert(X_COPIES * 8 * WW == X_ROWS, "");
  // Three workgroups on a CU, or two, or one.
  static constexpr int RING = OWN ? 64 * 1024 : kCuLds / (STAGE * 9 <= kCuLds ? 3 : STAGE * 6 <= kCuLds ? 2 : 1);
  static constexpr int FIT = RING / STAGE, MOST = 62 / COPIES + 2;
  static constexpr int STAGES = FIT < MOST ? FIT : MOST;
  static_assert(STAGES >= 3, "");
  static constexpr int JOIN = WAVES * RT * NT * 64 * 16;
  static constexpr int LDS = STAGES * STAGE > JOIN ? STAGES * STAGE : JOIN;
};

template <int DT>
__device__ __forceinline__ void round_row(const Q8Args& a, const char* raw, int8_t* codes, float* scale_out, uint32_t* tops) {
  const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6, units = (int)(a.pitch / 8);
  uint32_t top = 0;
  for (int u = threadIdx.x; u < units; u += blockDim.x) {
    float f[8];
    q8_load8<DT>(raw, u * 8, a.K, f);
#pragma unroll
    for (int i = 0; i < 8; ++i) top = q8_larger(top, __float_as_uint(f[i]) & 0x7fffffffu);
  }
  top = q8_largest(top);
  if ((threadIdx.x & 63) == 0) tops[wave] = top;
  __syncthreads();
  top = 0;
  for (int w = 0; w < waves; ++w) top = q8_larger(top, tops[w]);
  const float scale = q8_scale(top);
  if (threadIdx.x == 0) *scale_out = scale;
  const Q8Rounder rounder(scale);
  for (int u = threadIdx.x; u < units; u += blockDim.x) {
    float f[8];
    q8_load8<DT>(raw, u * 8, a.K, f);
    q8_store8(codes + u * 8, rounder, f);
  }
  __syncthreads();
}

// OWN: the one row of x is rounded here, by every workgroup for itself, while the first weights are on their way: a
// launch less (x 4096 x 4096: 9.4 -> 6.5 us).  Eight waves, as they share the rounding (four: 6.8).
template <int RT, int NT, int WW, int WAVES, bool OWN>
__global__ __launch_bounds__(64 * WAVES) void q8_few_kernel(const Q8Args a) {
  typedef Few<RT, NT, WW, WAVES, OWN> F;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int lane = threadIdx.x & 63, r16 = lane & 15, quarter = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave_w = wave % WW, part = wave / WW;
  // Neighbouring workgroups are on different XCDs: an XCD has every eighth tile of weights, for a group of slots one after
  // the other, so that the second slot of one matrix finds them in the XCD's L2.  Without spread all tiles of a slot follow
  // one another.
  const uint32_t block = blockIdx.x >> a.spread, chunk = divide_by(a.by_group, block), in_group = block - chunk * a.by_group.d;
  const uint32_t group = divide_by(a.by_tiles, chunk), eighth = chunk - group * a.by_tiles.d;
  const uint32_t slot = group * a.by_group.d + in_group, tile = (eighth << a.spread) + (blockIdx.x & ((1u << a.spread) - 1));
  if (tile >= a.tiles) return;
  int expert;
  uint32_t first, end;
  if (!find_tile(a, slot, 16 * NT, &expert, &first, &end)) return;
  const int pair = RT > 1 && a.glu ? 2 : 1;
  const int wave_cols = 16 * RT / pair;  // of y
  const int64_t wg_m0 = (int64_t)tile * (wave_cols * WW), m0 = wg_m0 + wave_w * wave_cols;
  if (expert == a.experts) {
    const uint32_t cols = wave_cols * WW;
    for (uint32_t i = threadIdx.x; i < F::X_ROWS * cols; i += 64 * WAVES) {
      const uint32_t n = first + i / cols;
      const int64_t m = wg_m0 + i % cols;
      if (n < end && m < a.out_rows) q8_store(a, n, m, 0.f);
    }
    return;
  }
  // Copies: eight rows at a time, eight lanes to a row.  A lane's 16 bytes go to its place in the row, so they come from
  // where that place's are: pieces are exchanged by half the row's number, for the operands' loads to find them on
  // different banks.
  const int row8 = lane >> 3;
  const int8_t* from[F::COPIES];
  uint32_t to[F::COPIES];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds + part * (F::ROWS * (int)kQ8Line);
#pragma unroll
  for (int i = 0; i < F::COPIES; ++i) {
    int row;  // of the part's rows in LDS
    if (i < 2 * RT) {
      const int r = i * 8 + row8;  // of the wave's weight rows
      row = wave_w * (16 * RT) + r;
      int64_t m = m0 + (pair == 2 ? r / 32 * 16 + r % 16 : r);
      m = m < a.out_rows ? m : a.out_rows - 1;
      if (pair == 2 && r % 32 >= 16) m += a.out_rows;
      from[i] = a.codes + ((int64_t)expert * a.M + m) * a.pitch;
    } else {
      const int r = ((i - 2 * RT) * WW + wave_w) * 8 + row8;
      row = F::W_ROWS + r;
      uint32_t n = first + r;
      n = n < end ? n : end - 1;
      from[i] = a.xq + q8_x_row(a, n) * a.pitch;
    }
    from[i] += ((lane & 7) ^ (row >> 1 & 7)) * 16;
    to[i] = lds0 + __builtin_amdgcn_readfirstlane(row - row8) * (int)kQ8Line;
  }
  // OWN: behind the ring the row's codes, then the row as it is, in whole KiB, then its scale and the waves' largest.
  char* codes = lds + F::LDS;
  const int raw_bytes = OWN ? a.K * (a.x_type == EBAG_F32 ? 4 : 2) : 0, chunks = (raw_bytes + 1023) / 1024;
  char* raw = codes + (OWN ? a.pitch : 0);
  float* own_scale = reinterpret_cast<float*>(raw + chunks * 1024);
  if (OWN) {
    for (int i = wave; i < chunks; i += WAVES) {
      const int at = i * 1024 + lane * 16;
      copy_to_lds((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)raw + i * 1024,
                  reinterpret_cast<const int8_t*>(a.x + (at < raw_bytes ? at : raw_bytes - 16)));
    }
  }
  const int lines = (int)(a.pitch / kQ8Line), steps = (lines + F::WK - 1) / F::WK, line0 = part * steps;
  // Not every workgroup begins with its first line: rows of a power of two bytes would have all of them ask the same
  // memory channels at a time (16 rows x 65536 x 8192: 117 us, like this 92; each eight neighbours, on an XCD each, alike, and the slots of a group).
  const int turn0 = (int)(chunk % (uint32_t)steps);
  auto line_of = [&](int step) { return line0 + (step + turn0 < steps ? step + turn0 : step + turn0 - steps); };
  auto copy = [&](int step, int stage) __attribute__((always_inline)) {
    const int at = line_of(step), line = at < lines ? at : lines - 1;  // one again where there is none
#pragma unroll
    for (int i = 0; i < F::COPIES; ++i) copy_to_lds(to[i] + stage * F::STAGE, from[i] + (int64_t)line * kQ8Line);
  };
  const char* mine = lds + part * (F::ROWS * (int)kQ8Line) + r16 * (int)kQ8Line;
  const int turn = r16 >> 1 & 7;
  i32x4 sum[RT][NT];
#pragma unroll
  for (int b = 0; b < RT; ++b)
#pragma unroll
    for (int t = 0; t < NT; ++t) sum[b][t] = i32x4{0, 0, 0, 0};
  const char* own_x = codes + quarter * 16;
  auto multiply = [&](int stage, int line) __attribute__((always_inline)) {
    const char* rows = mine + stage * F::STAGE;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int piece = ((h * 4 + quarter) ^ turn) * 16;
      i32x4 w[RT], x[NT];
#pragma unroll
      for (int b = 0; b < RT; ++b) w[b] = *reinterpret_cast<const i32x4*>(rows + (wave_w * RT + b) * (16 * (int)kQ8Line) + piece);
#pragma unroll
      for (int t = 0; t < NT; ++t)
        x[t] = *reinterpret_cast<const i32x4*>(OWN ? own_x + line * (int)kQ8Line + h * 64 : rows + (F::W_ROWS + 16 * t) * (int)kQ8Line + piece);
#pragma unroll
      for (int b = 0; b < RT; ++b)
#pragma unroll
        for (int t = 0; t < NT; ++t) sum[b][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x[t], w[b], sum[b][t], 0, 0, 0);
    }
  };
  for (int s = 0; s < F::STAGES - 1 && s < steps; ++s) copy(s, s);
  if (OWN) {
    if (steps >= F::STAGES - 1)
      arrived<(F::STAGES - 1) * F::COPIES>();
    else
      arrived<0>();
    uint32_t* tops = reinterpret_cast<uint32_t*>(own_scale + 1);
    int8_t* to_codes = reinterpret_cast<int8_t*>(codes);
    if (a.x_type == EBAG_F32)
      round_row<0>(a, raw, to_codes, own_scale, tops);
    else if (a.x_type == EBAG_F16)
      round_row<1>(a, raw, to_codes, own_scale, tops);
    else
      round_row<2>(a, raw, to_codes, own_scale, tops);
  }
  int stage = 0;
  for (int step = 0; step < steps; ++step) {
    // This step's copies are behind all but those of the STAGES - 2 steps after it, and every wave is done with the
    // stage before, which the next copies fill.
    if (step + F::STAGES - 2 < steps)
      arrived<(F::STAGES - 2) * F::COPIES>();
    else
      arrived<0>();
    const int before = stage ? stage - 1 : F::STAGES - 1;
    if (step + F::STAGES - 1 < steps) copy(step + F::STAGES - 1, before);
    if (line_of(step) < lines) multiply(stage, line_of(step));
    stage = stage + 1 < F::STAGES ? stage + 1 : 0;
  }
  // A lane has weight row r16 and rows 4 quarter .. of x.  The first of the waves that share columns finishes what all have.
  if (F::WK > 1) {
    __syncthreads();
    i32x4* joined = reinterpret_cast<i32x4*>(lds);
    if (part) {
#pragma unroll
      for (int b = 0; b < RT; ++b)
#pragma unroll
        for (int t = 0; t < NT; ++t) joined[((wave * RT + b) * NT + t) * 64 + lane] = sum[b][t];
    }
    __syncthreads();
    if (part) return;
#pragma unroll
    for (int p = 1; p < F::WK; ++p)
#pragma unroll
      for (int b = 0; b < RT; ++b)
#pragma unroll
        for (int t = 0; t < NT; ++t) sum[b][t] += joined[(((wave + p * WW) * RT + b) * NT + t) * 64 + lane];
  }
  const float* scales = a.scales + (int64_t)expert * a.M;
#pragma unroll
  for (int b = 0; b < RT; ++b) {
    if (pair == 2 && b % 2) continue;
    const int64_t m = m0 + (pair == 2 ? b / 2 : b) * 16 + r16;
    if (m >= a.out_rows) continue;
    const float ws = scales[m], wu = pair == 2 ? scales[a.out_rows + m] : 0.f;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t n = first + 16 * t + 4 * quarter + i;
        if (n >= end) continue;
        const float xs = OWN ? *own_scale : a.xs[q8_x_row(a, n)];
        float v = (float)sum[b][t][i] * (xs * ws);
        if (RT > 1 && pair == 2) {
          const float up = (float)sum[b + 1 < RT ? b + 1 : b][t][i] * (xs * wu);
          v = (a.y_type == EBAG_F32 ? q8_silu<true>(v) : q8_silu<false>(v)) * up;
        }
        q8_store(a, n, m, v);
      }
  }
}

template <int RT, int NT, int WW, int WAVES>
void launch(const Q8Args& a, unsigned grid, hipStream_t stream) {
  hipLaunchKernelGGL((q8_few_kernel<RT, NT, WW, WAVES, false>), dim3(grid), dim3(64 * WAVES), (Few<RT, NT, WW, WAVES, false>::LDS), stream, a);
}

constexpr int64_t kOwnTiles = 1024;  // of 16 rows of weights
int own_bytes(const Q8Args& a) {  // of LDS, behind the ring
  const int raw = a.K * (a.x_type == EBAG_F32 ? 4 : 2);
  return (int)a.pitch + (raw + 1023) / 1024 * 1024 + 4 * (1 + kQ8OwnWaves);
}

template <int RT, int WW>
void launch_own(const Q8Args& a, unsigned grid, hipStream_t stream) {
  constexpr int WAVES = kQ8OwnWaves / RT;
  hipLaunchKernelGGL((q8_few_kernel<RT, 1, WW, WAVES, true>), dim3(grid), dim3(64 * WAVES), (Few<RT, 1, WW, WAVES, true>::LDS) + own_bytes(a),
                     stream, a);
}

template <int RT>
void launch(const Q8Args& a, int x_tiles, int waves, unsigned grid, hipStream_t stream) {
  switch (x_tiles * 16 + waves) {
    case 16 + 1: return launch<RT, 1, 1, 4>(a, grid, stream);
    case 16 + 2: return launch<RT, 1, 2, 4>(a, grid, stream);
    case 32 + 1: return launch<RT, 2, 1, 4>(a, grid, stream);
    case 32 + 2: return launch<RT, 2, 2, 4>(a, grid, stream);
    case 32 + 4: return launch<RT, 2, 4, 4>(a, grid, stream);
    case 64 + 1: return launch<RT, 4, 1, 4>(a, grid, stream);
    case 64 + 2: return launch<RT, 4, 2, 4>(a, grid, stream);
    case 64 + 4: return launch<RT, 4, 4, 4>(a, grid, stream);
    case 64 + 8: return launch<RT, 4, 8, 8>(a, grid, stream);
    case 128 + 4: return launch<RT, 8, 4, 4>(a, grid, stream);
    default: return launch<RT, 8, 8, 8>(a, grid, stream);
  }
}

}  // namespace

// What the ring leaves of a CU's LDS, and x as copies take it.  With more workgroups than are on the card at a time their
// rounding costs more than the launch (bf16, in us, rounded here and first: 16384 x 4096 13.0, 17.3; 32768 x 160 10.0, 6.2; 32768
// x 8192 56.9, 53.0; 65536 x 8192 107, 95); so does a second row (16384 x 4096 18.9, 17.9; 4096 x 8192 13.5, 12.1; 4096 x 4096
// 8.8, 9.4).
bool q8_own_fits(const Q8Args& a) {
  const int elt = a.x_type == EBAG_F32 ? 4 : 2;
  return a.x && a.rows == 1 && !a.offsets && a.out_rows <= 16 * kOwnTiles && (int64_t)a.K * elt % 16 == 0 &&
         reinterpret_cast<uintptr_t>(a.x) % 16 == 0 && own_bytes(a) <= kCuLds - 64 * 1024;
}

void launch_q8_own(const Q8Args& a, int tiles, int waves, unsigned grid, hipStream_t stream) {
  if (tiles == 1)
    waves == 1 ? launch_own<1, 1>(a, grid, stream) : launch_own<1, 2>(a, grid, stream);
  else
    waves == 1 ? launch_own<2, 1>(a, grid, stream) : launch_own<2, 2>(a, grid, stream);
}

void launch_q8_few(const Q8Args& a, int tiles, int x_tiles, int waves, unsigned grid, hipStream_t stream) {
  tiles == 1 ? launch<1>(a, x_tiles, waves, grid, stream) : launch<2>(a, x_tiles, waves, grid, stream);
}

}  // namespace ebag
