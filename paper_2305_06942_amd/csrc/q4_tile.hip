// Products with 4-bit weights for many rows of x: the matrix-product kernel.
#include <hip/hip_runtime.h>

#include "gemv_ar.h"
#include "lanes.h"
#include "q4.h"
#include "q4_rows.h"

namespace ebag {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kStep = 128;   // columns of a step
constexpr int kB = 2;        // a wave's tiles of 32 weight rows

template <int DT>
__device__ __forceinline__ f32x16 mfma32(const vec16& a, const vec16& b, const f32x16& c) {
  if (DT == 1)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Sum of the eight elements of a vector.
template <int DT>
__device__ __forceinline__ float sum8(const vec16& v) {
  if (DT == 2) {
    const bf16x2 ones = __builtin_bit_cast(bf16x2, 0x3F803F80u);
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t two = v[i];
      s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), ones, s, false);
    }
    return s;
  }
  float f[8];
  Type<DT>::widen(v, f);
  return ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
}

// A float as the first three elements of a vector, exactly: three bf16 of 8 bits each, with
// fp16 x too, whose range ends at 65504 where a sum of its elements goes on.
__device__ __forceinline__ vec16 three_parts(float f) {
  typedef Type<2> T;
  uint32_t p[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const T::elt e = T::narrow(f);
    p[i] = __builtin_bit_cast(uint16_t, e);
    f -= T::widen(e);
  }
  return vec16{p[0] | p[1] << 16, p[2], 0, 0};
}

// WHOLE: a group is a multiple of 128 columns, so a step has one scale; otherwise
// every block of 32 columns has its own (fp16 and bf16: only with 64 rows of x, as with
// 32 the kernel for few rows is never slower; fp32: only 32, whose three parts fill LDS).
template <int DT, int NT, bool WHOLE, bool Y32>
struct Tile {
  static constexpr int BN = 32 * NT;                  // rows of x
  static constexpr int GROUPS = WHOLE ? 1 : 4;        // of a step
  static constexpr int PARTS = Q4Type<DT>::PARTS, VECS = DT == 0 ? 2 : 1, ELT = sizeof(typename Type<DT>::elt);
  static constexpr int PITCH = Y32 || WHOLE ? 272 : 336;  // bytes of a row of x in LDS: 16 lanes' vectors on different banks
  static constexpr int PART = BN * PITCH;             // of one part of fp32 x
  static constexpr int STAGED = BN * 16 / kThreads;   // vectors of a thread
};

// A workgroup has 256 rows of weights and BN = 32 NT rows of x, a wave 64 of the
// weight rows and all rows of x.  x goes through LDS, two steps of 128 columns in
// turn; a wave's codes come straight from memory, a step ahead, are made 16-bit
// numbers BASE + q in registers and are multiplied from there, so every weight is
// unpacked once for BN rows.  A group's sums start at zero, are corrected for BASE
// and the zero point, and are added to the tile's sums times the scale.  The
// correction, -(BASE + zero) * (sum of x), is one more matrix instruction, in bf16: the
// sum of x is found when x is staged and lies behind its row in three parts, whose
// sum is exact, and the other operand is -(BASE + zero) three times.  With fp32 y (Y32) BASE
// and zero come off the codes, three vector instructions for every pair of bf16 codes and
// one for fp16's, and there is no correction (2048 x 8192 x 4096 with fp32 and 16-bit y:
// bf16 235 and 158 us, fp16 161 and 165); three parts of fp32 x are multiplied with the
// codes (2048 x 4096 x 4096: 234 us, 294 TFLOP/s, 880 of the matrix unit's; fp32's own
// 154).
//
// Bound by the latency and the L1 work of its loads: 32768 rows on 64 experts of 4096 x
// 2048 (550 GFLOP) 740 us, 745 TFLOP/s, from about the thirtieth launch on (on an idle
// card the first ones take up to 1000); a large bf16 product reaches 1360.  The
// same loads from one hot place 630 us, without loads 494, of which a ninth is the
// correction.  512 weight rows to a workgroup (one on a CU instead of two) take 921 us;
// 32 rows of x 1073.  256 x 64 is what the registers hold twice on a CU: 128 of 256 of a
// lane are sums.
//
// WORDS: rows of codes begin at multiples of 4 bytes.  Others are loaded from the
// multiple of 4 below and shifted in registers (32768 rows on 64 experts of 4096 x
// 2044, rows of 1022 bytes: 1241 us loaded at their own addresses, 904 us shifted).
template <int DT, int NT, bool WHOLE, bool ZEROS, bool WORDS, bool Y32>
__global__ __launch_bounds__(kThreads, 2) void q4_tile_kernel(const Q4Args a) {
  typedef Tile<DT, NT, WHOLE, Y32> C;
  typedef Type<DT> T;
  typedef Q4Type<DT> Q;
  __shared__ __attribute__((aligned(16))) char lds[2][C::PARTS * C::PART];
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, r32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t slot = divide_by(a.by_tiles, blockIdx.x), tile = blockIdx.x - slot * a.by_tiles.d;
  int expert;
  uint32_t first, end;
  if (!find_tile(a, slot, C::BN, &expert, &first, &end)) return;
  // Rows of weights: with glu, a wave's two tiles are gate rows and the up rows that go with them.
  const int pair = a.glu ? 2 : 1;
  const int64_t wg_m0 = (int64_t)tile * (32 * kB * kWaves / pair);
  if (expert == a.experts) {
    const uint32_t cols = 32 * kB * kWaves / pair;
    for (uint32_t i = tid; i < C::BN * cols; i += kThreads) {
      const uint32_t n = first + i / cols;
      const int64_t m = wg_m0 + i % cols;
      if (n < end && m < a.out_rows) store_y<DT, Y32>(a, n, m, 0.f);
    }
    return;
  }
  const int64_t m0 = wg_m0 + wave * (32 * kB / pair);
  // Uniform addresses of the wave's first row of each tile, and a lane's 32-bit distances from them.
  const uint8_t* codes[kB];
  const char* scales[kB];
  const uint8_t* zeros[kB];
  uint32_t codes_at[kB], group_at[kB], shift[kB];
#pragma unroll
  for (int b = 0; b < kB; ++b) {
    const int64_t from = m0 + (pair == 2 ? 0 : 32 * b);  // may lie behind the last row: then all lanes take that one
    const int64_t base = from < a.out_rows ? from : a.out_rows - 1;
    int64_t m = from + r32;
    m = m < a.out_rows ? m : a.out_rows - 1;
    const int64_t row = base + (pair == 2 && b ? a.out_rows : 0) + (int64_t)expert * a.M;
    codes[b] = a.codes + row * a.row_bytes;
    scales[b] = a.scales + row * a.groups * C::ELT;
    zeros[b] = a.zeros ? a.zeros + row * a.groups : nullptr;
    codes_at[b] = (uint32_t)(m - base) * (uint32_t)a.row_bytes + half * 16;
    if (!WORDS) {
      const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(codes[b]) & 3);
      codes[b] -= off;
      codes_at[b] += off;
      shift[b] = codes_at[b] & 3;
      codes_at[b] -= shift[b];
    }
    group_at[b] = (uint32_t)(m - base) * (uint32_t)a.groups;
  }
  // Staging: thread (row, chunk) has vector `chunk` of rows row, row + 16, ...
  const int chunk = tid & 15;
  const char* x[C::STAGED];
#pragma unroll
  for (int i = 0; i < C::STAGED; ++i) {
    uint32_t n = first + (tid >> 4) + 16 * i;
    n = n < end ? n : end - 1;
    int64_t row = a.src ? (int64_t)divide_by(a.by_choices, (uint32_t)a.src[n] & 0x7fffffffu) : (int64_t)n;
    row = row < a.x_rows ? row : a.x_rows - 1;
    x[i] = a.x + row * a.ldx + chunk * (8 * C::ELT);
  }

  struct Weights {
    vec16 w[kB][2];  // bytes half * 16 .. of each 32: word j has columns 64 i + 32 half + 8 j
    typename T::elt scale[kB][C::GROUPS];
    uint32_t zero[kB][C::GROUPS];
    uint32_t behind[kB];  // not WORDS: the word behind the row's last one here
  };
  // tail: the step passes the end of K.
  auto load_weights = [&](Weights& o, int step, bool tail) {
#pragma unroll
    for (int b = 0; b < kB; ++b)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint8_t* base = codes[b] + (int64_t)step * (kStep / 2) + 32 * i;
        o.w[b][i] = !tail   ? load16(reinterpret_cast<const char*>(base) + codes_at[b])
                    : WORDS ? load_codes_end(a, base + codes_at[b])
                            : load_words_end(a, base + codes_at[b]);
      }
    if (!WORDS) {
#pragma unroll
      for (int b = 0; b < kB; ++b) {
        const uint8_t* row = codes[b] + (int64_t)step * (kStep / 2) + (codes_at[b] - 16 * half);
        const uint8_t* p = tail ? word_behind(row, kStep / 2, shift[b], a.codes + a.codes_bytes)
                                : row + (kStep / 2 - (shift[b] ? 0 : 4));
        o.behind[b] = *reinterpret_cast<const uint32_t*>(p);
      }
    }
#pragma unroll
    for (int g = 0; g < C::GROUPS; ++g) {
      uint32_t at = divide_by(a.by_group_blocks, (uint32_t)(step * 4 + g));
      if (tail) at = at < (uint32_t)a.groups ? at : a.groups - 1;
#pragma unroll
      for (int b = 0; b < kB; ++b) {
        o.scale[b][g] = *reinterpret_cast<const typename T::elt*>(scales[b] + C::ELT * at + C::ELT * group_at[b]);
        o.zero[b][g] = ZEROS ? *(zeros[b] + at + group_at[b]) : 8u;
      }
    }
  };
  auto load_rows = [&](vec16 (*v)[C::VECS], int step, bool tail) {
    if (!tail) {
#pragma unroll
      for (int i = 0; i < C::STAGED; ++i)
#pragma unroll
        for (int j = 0; j < C::VECS; ++j) v[i][j] = load16(x[i] + (int64_t)step * (kStep * C::ELT) + 16 * j);
      return;
    }
    const int n = a.K - step * kStep - 8 * chunk;  // elements left
#pragma unroll
    for (int i = 0; i < C::STAGED; ++i) load_x<DT>(x[i] + (int64_t)step * (kStep * C::ELT), n, a.K, v[i]);
  };
  auto store_rows = [&](const vec16 (*v)[C::VECS], char* to) {
    char* row = to + (tid >> 4) * C::PITCH;
    if constexpr (DT == 0) {
#pragma unroll
      for (int i = 0; i < C::STAGED; ++i) {
        vec16 parts[C::PARTS];
        split_f32(v[i][0], v[i][1], parts);
#pragma unroll
        for (int p = 0; p < C::PARTS; ++p)
          *reinterpret_cast<vec16*>(row + p * C::PART + 16 * i * C::PITCH + chunk * 16) = parts[p];
      }
    } else if constexpr (Y32) {
#pragma unroll
      for (int i = 0; i < C::STAGED; ++i)
        *reinterpret_cast<vec16*>(row + 16 * i * C::PITCH + chunk * 16) = pair_order(v[i][0]);
    } else {
      // Lane `chunk` of a row (or of a quarter of it) finishes the sums of row number `chunk` % STAGED.
      float mine = 0.f;
      const int pick = (WHOLE ? chunk : chunk & 3) % C::STAGED;
#pragma unroll
      for (int i = 0; i < C::STAGED; ++i) {
        const float s = sum_lanes(sum8<DT>(v[i][0]), WHOLE ? 16 : 4);
        mine = i == pick ? s : mine;
        *reinterpret_cast<vec16*>(row + 16 * i * C::PITCH + chunk * 16) = pair_order(v[i][0]);
      }
      if ((WHOLE ? chunk : chunk & 3) < C::STAGED)
        *reinterpret_cast<vec16*>(row + 16 * pick * C::PITCH + 256 + (WHOLE ? 0 : chunk / 4 * 16)) = three_parts(mine);
    }
  };

  const CodeBits<DT, Y32> bits;
  f32x16 sum[kB][NT];
#pragma unroll
  for (int b = 0; b < kB; ++b)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) sum[b][t][i] = 0.f;

  Weights now, next;
  vec16 staged[C::STAGED][C::VECS];
  enum Next { WHOLE_STEP, TAIL_STEP, NONE };
  // One step's products; what the next one needs is loaded ahead of them and staged behind.
  auto work = [&](int step, Next after) __attribute__((always_inline)) {
    if (after != NONE) {
      load_weights(next, step + 1, after == TAIL_STEP);
      load_rows(staged, step + 1, after == TAIL_STEP);
    }
    const char* from = lds[step & 1] + r32 * C::PITCH;
    if (!WORDS) {
      // The word after a lane's four: the other half's first one, of the same 32 bytes or of the next.
#pragma unroll
      for (int b = 0; b < kB; ++b) {
        const u32x2 both = __builtin_amdgcn_permlane32_swap(now.w[b][0][0], now.w[b][1][0], false, false);
        const u32x2 upper = __builtin_amdgcn_permlane32_swap(now.w[b][1][0], now.w[b][1][0], false, false);
        const uint32_t after[2] = {half ? both[0] : both[1], half ? now.behind[b] : upper[1]};
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            now.w[b][i][j] = __builtin_amdgcn_alignbyte(j < 3 ? now.w[b][i][j < 3 ? j + 1 : 3] : after[i], now.w[b][i][j], shift[b]);
      }
    }
#pragma unroll
    for (int b = 0; b < kB; ++b)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 4; j += 2) {  // columns 8 half .. of 16 in both halves
          const u32x2 s = __builtin_amdgcn_permlane32_swap(now.w[b][i][j], now.w[b][i][j + 1], false, false);
          now.w[b][i][j] = s[0];
          now.w[b][i][j + 1] = s[1];
        }
    constexpr int SLICES = 8 / C::GROUPS;  // of 16 columns, of a group
#pragma unroll
    for (int g = 0; g < C::GROUPS; ++g) {
      f32x16 v[kB][NT];
#pragma unroll
      for (int sl = 0; sl < SLICES; ++sl) {
        const int slice = g * SLICES + sl;
        vec16 xs[NT][C::PARTS];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int p = 0; p < C::PARTS; ++p)
            xs[t][p] = *reinterpret_cast<const vec16*>(from + p * C::PART + 32 * t * C::PITCH + slice * 32 + half * 16);
#pragma unroll
        for (int b = 0; b < kB; ++b) {
          // Of each 64 columns, words 0 and 2 have the first 32, words 1 and 3 the others.
          vec16 q = unpack_codes(bits, now.w[b][slice / 4][slice % 4 / 2 + 2 * (slice % 2)]);
          if constexpr (Y32) q = centred(bits, q, -Q::BASE - (float)now.zero[b][g]);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            if (sl == 0)
#pragma unroll
              for (int i = 0; i < 16; ++i) v[b][t][i] = 0.f;
#pragma unroll
            for (int p = 0; p < C::PARTS; ++p) v[b][t] = mfma32<DT>(xs[t][p], q, v[b][t]);
          }
        }
      }
      vec16 xsum[NT];
      if (!Y32) {
#pragma unroll
        for (int t = 0; t < NT; ++t) xsum[t] = *reinterpret_cast<const vec16*>(from + 32 * t * C::PITCH + 256 + g * 16);
      }
#pragma unroll
      for (int b = 0; b < kB; ++b) {
        const float scale = T::widen(now.scale[b][g]);
        if constexpr (!Y32) {
          const uint32_t o = __builtin_bit_cast(uint16_t, Type<2>::narrow(-Q::BASE - (float)now.zero[b][g]));  // 143 at most: 8 bits
          const vec16 off = {half ? 0u : o | o << 16, half ? 0u : o, 0, 0};
#pragma unroll
          for (int t = 0; t < NT; ++t) v[b][t] = mfma32<2>(xsum[t], off, v[b][t]);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int i = 0; i < 16; ++i) sum[b][t][i] = __builtin_fmaf(scale, v[b][t][i], sum[b][t][i]);
      }
      if (!WHOLE) __builtin_amdgcn_sched_barrier(0);  // one group's sums at a time: registers
    }
    if (after != NONE) {
      store_rows(staged, lds[(step + 1) & 1]);
      now = next;
      __syncthreads();
    }
  };
  const int whole = a.K / kStep, steps = (a.K + kStep - 1) / kStep;
  load_rows(staged, 0, whole == 0);
  load_weights(now, 0, whole == 0);
  store_rows(staged, lds[0]);
  __syncthreads();
  int step = 0;
  for (; step + 1 < whole; ++step) work(step, WHOLE_STEP);
  if (step + 1 < steps) work(step++, TAIL_STEP);
  work(step, NONE);
  // A lane has weight row r32 and, in element i, row 8 (i / 4) + 4 half + i % 4 of x.
#pragma unroll
  for (int b = 0; b < kB; ++b) {
    if (pair == 2 && b) continue;
    const int64_t m = m0 + 32 * b + r32;
    if (m >= a.out_rows) continue;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const uint32_t n = first + 32 * t + 8 * (i / 4) + 4 * half + i % 4;
        if (n < end) store_y<DT, Y32>(a, n, m, pair == 2 ? silu<Y32>(sum[0][t][i]) * sum[1][t][i] : sum[b][t][i]);
      }
  }
}

typedef void (*tile_fn)(const Q4Args);

template <int DT, int NT, bool WHOLE, bool Y32>
tile_fn pick(bool zeros, bool words) {
  if (words) return zeros ? q4_tile_kernel<DT, NT, WHOLE, true, true, Y32> : q4_tile_kernel<DT, NT, WHOLE, false, true, Y32>;
  return zeros ? q4_tile_kernel<DT, NT, WHOLE, true, false, Y32> : q4_tile_kernel<DT, NT, WHOLE, false, false, Y32>;
}

template <int DT, bool Y32>
tile_fn pick(int x_tiles, bool whole, bool zeros, bool words) {
  if (!whole) return pick<DT, 2, false, Y32>(zeros, words);
  return x_tiles == 1 ? pick<DT, 1, true, Y32>(zeros, words) : pick<DT, 2, true, Y32>(zeros, words);
}

}  // namespace

void launch_q4_tile(const Q4Args& a, int dtype, bool y32, int x_tiles, unsigned grid, hipStream_t stream) {
  const bool whole = a.group % 128 == 0, zeros = a.zeros != nullptr;
  const bool words = a.row_bytes % 4 == 0 && reinterpret_cast<uintptr_t>(a.codes) % 4 == 0;
  const tile_fn fn = dtype == EBAG_F16    ? y32 ? pick<1, true>(x_tiles, whole, zeros, words) : pick<1, false>(x_tiles, whole, zeros, words)
                     : dtype == EBAG_BF16 ? y32 ? pick<2, true>(x_tiles, whole, zeros, words) : pick<2, false>(x_tiles, whole, zeros, words)
                     : whole              ? pick<0, 1, true, true>(zeros, words)
                                          : pick<0, 1, false, true>(zeros, words);
  hipLaunchKernelGGL(fn, dim3(grid), dim3(kThreads), 0, stream, a);
}

}  // namespace ebag
