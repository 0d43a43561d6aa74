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
  Divisor by_choices;
  Divisor by_group_blocks;  // group / 32
  Divisor by_tiles;         // workgroups that share the rows of x, each with its rows of weights
  // The kernel for few rows.
  int32_t split;            // waves that share a tile
  int32_t turns;            // tiles that a wave works through
  int32_t x_bytes;          // LDS for x; the waves' sums lie behind
  int32_t all_columns;      // K in whole units
  int32_t some_columns;     // columns of 16 rows of x that fit, in whole units for each of a tile's waves
  int32_t fit_rows;         // rows of x that fit with all their columns
  Divisor by_all, by_some;  // those columns / 8
};

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// A weight's code q goes through the matrix instructions as BASE + q, which is a
// bit pattern away in fp16 and bf16 (BASE is a power of two with q at the bottom
// of its mantissa, or above it) and exact; BASE and the zero point come off again
// as (BASE + zero) * (the sum of x over the group).  The sums grow by BASE / 8 at
// most that way, so fp32 loses 3 bits (fp16) or 4 (bf16) of its 24: fewer than the
// rounding of y to 11 and 8 bits does, and the larger BASE leaves one code of
// four where it is and saves its shift.  An fp32 y keeps all its bits, so there BASE +
// zero comes off each code before the products (`centred`; Y32 in the kernels; one row x
// 65536 x 8192: bf16 57 us with a bf16 y, 77 with fp32, fp16 61 and 62).  fp32 x
// goes as three bf16 parts whose sum is x, bit for bit (but for bits below 2^-133), so
// its products are exact too.
template <int DT> struct Q4Type;

template <> struct Q4Type<1> {
  static constexpr int PARTS = 1;
  static constexpr uint32_t ONES = 0x3C003C00u;
  static constexpr float BASE = 64.f;
  static constexpr uint32_t MASK = 0x00F000F0u, HIGH = 0x54005400u;
  // Codes j and j + 4 of a word of eight (low bits first), under MASK.
  static __device__ __forceinline__ uint32_t pair(uint32_t w, int j) { return j == 0 ? w << 4 : w >> (4 * (j - 1)); }
  static __device__ __forceinline__ f32x4 mfma(const vec16& a, const vec16& b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};

template <> struct Q4Type<2> {
  static constexpr int PARTS = 1;
  static constexpr uint32_t ONES = 0x3F803F80u;
  static constexpr float BASE = 128.f;
  static constexpr uint32_t MASK = 0x000F000Fu, HIGH = 0x43004300u;
  static __device__ __forceinline__ uint32_t pair(uint32_t w, int j) { return w >> (4 * j); }
  static __device__ __forceinline__ f32x4 mfma(const vec16& a, const vec16& b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};

template <> struct Q4Type<0> : Q4Type<2> {
  static constexpr int PARTS = 3;
};

// MASK and HIGH in registers: as literals they would take an instruction each,
// and from one scalar and one vector register both go into one.  For `centred` bf16
// codes 1 in the lower and in the upper half, too (as an inline constant 1.0 stands in
// the upper one).
template <int DT, bool Y32>
struct CodeBits {
  uint32_t mask, high, lower, upper;
  __device__ __forceinline__ CodeBits() {
    asm volatile("s_mov_b32 %0, %1" : "=s"(mask) : "i"(Q4Type<DT>::MASK));
    asm volatile("v_mov_b32 %0, %1" : "=v"(high) : "i"(Q4Type<DT>::HIGH));
    if (Y32 && DT != 1) {
      asm volatile("s_mov_b32 %0, 0x3f80" : "=s"(lower));
      asm volatile("s_mov_b32 %0, 0x3f800000" : "=s"(upper));
    }
  }
};

// Eight codes of a word as BASE + q, in the order 0 4, 1 5, 2 6, 3 7.
template <int DT, bool Y32>
__device__ __forceinline__ vec16 unpack_codes(const CodeBits<DT, Y32>& c, uint32_t w) {
  vec16 r;
#pragma unroll
  for (int j = 0; j < 4; ++j) r[j] = (Q4Type<DT>::pair(w, j) & c.mask) | c.high;
  return r;
}

// Eight numbers BASE + q with off = -(BASE + zero) added: q - zero, exact.  fp16: two at
// a time.  bf16: a dot product with (1, 0) or (0, 1) widens one of two and adds in one
// instruction.
template <int DT>
__device__ __forceinline__ vec16 centred(const CodeBits<DT, true>& c, const vec16& codes, float off) {
  vec16 r;
  if (DT == 1) {
    const f16x2 both = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_pkrtz(off, off));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t two = codes[j];
      r[j] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, two) + both);
    }
    return r;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t two = codes[j];
    const float lo = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, c.lower), __builtin_bit_cast(bf16x2, two), off, false);
    const float hi = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, c.upper), __builtin_bit_cast(bf16x2, two), off, false);
    r[j] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
  }
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

// A vector without its first `bytes` (0 to 15), zeros behind.
__device__ __forceinline__ vec16 without_first(const vec16& v, int bytes) {
  uint64_t lo = v[0] | (uint64_t)v[1] << 32, hi = v[2] | (uint64_t)v[3] << 32;
  if (bytes >= 8) {
    lo = hi;
    hi = 0;
  }
  const int s = 8 * (bytes & 7);
  if (s) lo = lo >> s | hi << (64 - s);
  hi >>= s;
  return vec16{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}

// 16 bytes of codes; what lies behind a row's end is not used, what lies
// behind the last matrix is not read.
__device__ __forceinline__ vec16 load_codes_end(const Q4Args& a, const uint8_t* p) {
  const int64_t left = a.codes + a.codes_bytes - p;
  if (left >= 16) return load16(reinterpret_cast<const char*>(p));
  if (left <= 0) return vec16{0, 0, 0, 0};
  if (a.codes_bytes >= 16) return without_first(load16(reinterpret_cast<const char*>(p + left - 16)), 16 - (int)left);
  vec16 r = {0, 0, 0, 0};
  for (int i = 0; i < left; ++i) r[i / 4] |= (uint32_t)p[i] << (8 * (i % 4));
  return r;
}

// The same at a multiple of 4 bytes, in whole words: one is read if a byte of it is
// in range, and zero otherwise.
__device__ __forceinline__ vec16 load_words_end(const Q4Args& a, const uint8_t* p) {
  vec16 r = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (p + 4 * i < a.codes + a.codes_bytes) r[i] = reinterpret_cast<const uint32_t*>(p)[i];
  return r;
}

// The first n (at most 8) of eight elements of a row of x of K, zeros behind them.
template <int DT>
__device__ __forceinline__ void load_x(const char* p, int n, int K, vec16* v) {
  constexpr int VECS = DT == 0 ? 2 : 1, N = DT == 0 ? 4 : 8, ELT = 16 / N;
#pragma unroll
  for (int i = 0; i < VECS; ++i) {
    const int have = n - i * N;
    const char* at = p + 16 * i;
    v[i] = vec16{0, 0, 0, 0};
    if (have >= N)
      v[i] = load16(at);
    else if (have > 0 && K >= N)  // the row's last vector, without what is before `at`
      v[i] = without_first(load16(at + have * ELT - 16), 16 - have * ELT);
    else if (have > 0)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        if (e >= have) continue;
        if (DT == 0)
          v[i][e % 4] = reinterpret_cast<const uint32_t*>(at)[e];
        else
          v[i][e / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(at)[e] << (16 * (e % 2));
      }
  }
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

template <int DT, bool Y32>
__device__ __forceinline__ void store_y(const Q4Args& a, uint32_t n, int64_t m, float v) {
  typedef Type<DT> T;
  char* p = a.y + n * a.ldy;
  if (Y32)
    reinterpret_cast<float*>(p)[m] = v;
  else
    reinterpret_cast<typename T::elt*>(p)[m] = T::narrow(v);
}

// v / (1 + exp(-v)).  With the short exponential, off by (|v| + 8) 2^-22, where y is rounded
// to 16 bits; an fp32 y gets the full one, of -|v|, which does not overflow where the
// result is still a number.
template <bool Y32>
__device__ __forceinline__ float silu(float v) {
  if (!Y32) return v / (1.f + __expf(-v));
  const float e = expf(-fabsf(v));
  return v * ((v < 0.f ? e : 1.f) / (1.f + e));
}

typedef void (*q4_fn)(const Q4Args);

// Which instance of the kernel for few rows a launch takes.
struct Q4FewKind {
  int tiles;    // of 16 weight rows of a wave: 1, or 2 with glu
  bool whole;   // a group is a multiple of 128 columns
  bool zeros;   // there are zero points
  bool words;   // rows of codes begin at multiples of 4 bytes
  bool y32;     // y is fp32
};
q4_fn pick_q4_few_f32(const Q4FewKind& k);
q4_fn pick_q4_few_f16(const Q4FewKind& k);
q4_fn pick_q4_few_bf16(const Q4FewKind& k);

// The matrix-product kernel for many rows of x: a workgroup for
// kQ4TileRows rows of weights (half as many outputs with glu) and 32 x_tiles (1 or
// 2; fp32: 1) rows of x.
constexpr int kQ4TileRows = 256;
void launch_q4_tile(const Q4Args& a, int dtype, bool y32, int x_tiles, unsigned grid, hipStream_t stream);

}  // namespace ebag
