// Products with 4-bit weights (gemv_ar_q4_* of include/gemv_ar.h): rounding to 4
// bits, and the kernel for few rows of x.
#include <hip/hip_runtime.h>

#include <climits>
#include <new>

#include "ebag_a2a.h"
#include "gemv_ar.h"
#include "lanes.h"
#include "q4.h"

using namespace ebag;

namespace {

// ------------------------------------------------------------------- few rows
//
// A workgroup has RT tiles of 16 rows of weights and 16 rows of x; its
// waves split K in units of 256 columns (a cache line of codes), wave w
// taking units w, w + waves, ..., and join their sums in LDS at the end.  A
// lane loads 16 bytes, 32 consecutive codes of row lane % 16; a transposition
// between the four lanes of a row (lane / 16) then gives word t of each the
// columns 32 t + 8 (lane / 16) .. + 8, the layout of a 16x16x32 matrix
// instruction over 32 consecutive columns, which belong to one group.  x is
// the first operand, so a lane holds sums of ONE weight row for four rows of x
// and needs one scale per group: the four lanes of a row load those of four
// blocks of 32 columns and pass them round.  Rows of a tile beyond the last one
// repeat it; nothing they give is stored.
//
// The loads of a wave's next unit are under way while it works on one.

// Between lanes l, l + 16, l + 32, l + 48: w[t] of lane quarter c becomes w[c] of quarter t.
__device__ __forceinline__ void transpose_words(vec16& w) {
  u32x2 s;
  s = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
  w[0] = s[0]; w[2] = s[1];
  s = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
  w[1] = s[0]; w[3] = s[1];
  s = __builtin_amdgcn_permlane16_swap(w[0], w[1], false, false);
  w[0] = s[0]; w[1] = s[1];
  s = __builtin_amdgcn_permlane16_swap(w[2], w[3], false, false);
  w[2] = s[0]; w[3] = s[1];
}

// The words of the four quarters, in each of them.
__device__ __forceinline__ void gather_words(uint32_t w, uint32_t* all) {
  const u32x2 half = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  const u32x2 lo = __builtin_amdgcn_permlane16_swap(half[0], half[0], false, false);
  const u32x2 hi = __builtin_amdgcn_permlane16_swap(half[1], half[1], false, false);
  all[0] = lo[0]; all[1] = lo[1]; all[2] = hi[0]; all[3] = hi[1];
}

constexpr int kFewThreads = 512, kCuLds = 160 * 1024;

// What a launch is compiled for.  WHOLE: a group is a multiple of 128 columns, so
// a step of 128 has one scale.  ZEROS: there are zero points.
template <int DT_, int RT_, bool WHOLE_, bool ZEROS_>
struct FewShape {
  static constexpr int DT = DT_, RT = RT_;
  static constexpr bool WHOLE = WHOLE_, ZEROS = ZEROS_;
  static constexpr int STEPS = WHOLE ? 4 : 2;     // of a unit
  static constexpr int SCALES = WHOLE ? 1 : STEPS;  // loads of scales of a unit: four lanes of a row load one each
  static constexpr int COLUMNS = 128 * STEPS;
};

// Where a lane of a wave with RT tiles of weight rows loads its next unit from.
template <class C>
struct Few {
  const uint8_t* codes[C::RT];  // its row of weights, its quarter's bytes
  const char* scales[C::RT];    // that row's first scale
  const uint8_t* zeros[C::RT];  // and zero
  int unit, split;

  __device__ __forceinline__ void advance() {
#pragma unroll
    for (int rt = 0; rt < C::RT; ++rt) codes[rt] += split * (C::COLUMNS / 2);
    unit += split;
  }
};

// A unit's weights, as loaded.  WHOLE: a lane has the scale and zero of step
// `quarter`; otherwise those of block `quarter` of each step.
template <class C>
struct Unit {
  vec16 w[C::STEPS][C::RT];
  uint32_t scale[C::SCALES][C::RT], zero[C::SCALES][C::RT];
};

// END: the unit passes the end of K.
template <bool END, class C>
__device__ __forceinline__ void load_weights(const Q4Args& a, const Few<C>& f, Unit<C>& o) {
  const int quarter = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int s = 0; s < C::STEPS; ++s)
#pragma unroll
    for (int rt = 0; rt < C::RT; ++rt) {
      const uint8_t* p = f.codes[rt] + s * 64;
      o.w[s][rt] = END ? load_codes_end(a, p) : load16(reinterpret_cast<const char*>(p));
    }
#pragma unroll
  for (int s = 0; s < C::SCALES; ++s) {
    const int block = f.unit * (4 * C::STEPS) + (C::WHOLE ? 4 * quarter : 4 * s + quarter);
    uint32_t g = divide_by(a.by_group_blocks, (uint32_t)block);
    if (END) g = g < (uint32_t)a.groups ? g : a.groups - 1;
#pragma unroll
    for (int rt = 0; rt < C::RT; ++rt) {
      o.scale[s][rt] = C::DT == 0 ? reinterpret_cast<const uint32_t*>(f.scales[rt])[g]
                                  : (uint32_t)reinterpret_cast<const uint16_t*>(f.scales[rt])[g];
      o.zero[s][rt] = C::ZEROS ? f.zeros[rt][g] : 8u;
    }
  }
}

// The unit's products, added to the sums.  x: the lane's row of x in LDS, the
// unit's columns; the parts of fp32 x are `pitch` bytes apart.
template <class C>
__device__ __forceinline__ void multiply(const CodeBits<C::DT>& bits, Unit<C>& o, const char* x, int pitch, f32x4* sum) {
  typedef Q4Type<C::DT> Q;
  typedef Type<C::DT> T;
  constexpr int PARTS = Q::PARTS, RT = C::RT;
  constexpr bool F32 = C::DT == 0;
  const vec16 ones = {Q::ONES, Q::ONES, Q::ONES, Q::ONES};
  uint32_t all[RT][4], zero[RT][4];  // scale, and the zero above it or in a word of its own
#pragma unroll
  for (int s = 0; s < C::STEPS; ++s) {
    float scale[RT][4], off[RT][4];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      transpose_words(o.w[s][rt]);
      if (!C::WHOLE || s == 0) {
        gather_words(o.scale[s][rt] | (C::ZEROS && !F32 ? o.zero[s][rt] << 16 : 0u), all[rt]);
        if (C::ZEROS && F32) gather_words(o.zero[s][rt], zero[rt]);
      }
#pragma unroll
      for (int t = 0; t < (C::WHOLE ? 1 : 4); ++t) {
        const int at = C::WHOLE ? s : t;
        scale[rt][t] = F32 ? __uint_as_float(all[rt][at])
                           : T::widen(__builtin_bit_cast(typename T::elt, (typename Bits<C::DT>::type)all[rt][at]));
        off[rt][t] = C::ZEROS ? -Q::BASE - (float)(F32 ? zero[rt][at] : all[rt][at] >> 16) : -Q::BASE - 8.f;
      }
    }
    f32x4 v[RT], xsum;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      vec16 xs[PARTS];
#pragma unroll
      for (int p = 0; p < PARTS; ++p) xs[p] = *reinterpret_cast<const vec16*>(x + p * pitch + (s * 4 + t) * 64);
      if (!C::WHOLE || t == 0) xsum = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int p = 0; p < PARTS; ++p) xsum = Q::mfma(xs[p], ones, xsum);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const vec16 q = unpack_codes(bits, o.w[s][rt][t]);
        if (!C::WHOLE || t == 0) v[rt] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int p = 0; p < PARTS; ++p) v[rt] = Q::mfma(xs[p], q, v[rt]);
        if (C::WHOLE && t < 3) continue;
        const int g = C::WHOLE ? 0 : t;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          sum[rt][i] = __builtin_fmaf(scale[rt][g], __builtin_fmaf(off[rt][g], xsum[i], v[rt][i]), sum[rt][i]);
      }
    }
  }
}

// Rows first .. first + rows of x into LDS, columns k0 .. k0 + cols (by8: cols / 8),
// in pair order, zeros behind column K; row r at r * pitch, further parts of
// fp32 rows * pitch behind.
template <int DT>
__device__ __forceinline__ void stage_x(const Q4Args& a, uint32_t first, int rows, int k0, const Divisor& by8, int pitch,
                                        char* lds) {
  constexpr int ELT = DT == 0 ? 4 : 2, VECS = DT == 0 ? 2 : 1, PARTS = Q4Type<DT>::PARTS, AT_ONCE = 4;
  const uint32_t n = rows * by8.d;
  for (uint32_t i0 = threadIdx.x; i0 < n; i0 += AT_ONCE * blockDim.x) {
    vec16 v[AT_ONCE][VECS];
    char* to[AT_ONCE];
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      const uint32_t i = i0 + j * blockDim.x < n ? i0 + j * blockDim.x : n - 1;
      const uint32_t r = divide_by(by8, i), c = i - r * by8.d;
      int64_t row = a.src ? (int64_t)divide_by(a.by_choices, (uint32_t)a.src[first + r] & 0x7fffffffu) : (int64_t)(first + r);
      row = row < a.x_rows ? row : a.x_rows - 1;
      const int k = k0 + 8 * (int)c;
      load_x<DT>(a.x + row * a.ldx + (int64_t)k * ELT, a.K - k, a.K, v[j]);
      to[j] = lds + r * pitch + c * 16;
    }
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      vec16 parts[PARTS];
      if (DT == 0)
        split_f32(v[j][0], v[j][VECS - 1], parts);
      else
        parts[0] = pair_order(v[j][0]);
#pragma unroll
      for (int p = 0; p < PARTS; ++p) *reinterpret_cast<vec16*>(to[j] + p * rows * pitch) = parts[p];
    }
  }
}

template <class C>
__global__ __launch_bounds__(kFewThreads, C::RT == 1 ? 4 : 2) void q4_few_kernel(const Q4Args a) {
  constexpr int DT = C::DT, RT = C::RT;
  extern __shared__ __attribute__((aligned(16))) char lds[];  // x; the waves' sums [2][waves][RT][64]
  const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r16 = lane & 15, quarter = lane >> 4;
  const int tiles = waves / a.split, own = wave / a.split, part = wave - own * a.split;
  const uint32_t slot = divide_by(a.by_tiles, blockIdx.x);
  int expert;
  uint32_t first, end;
  if (!find_tile(a, slot, 16, &expert, &first, &end)) return;
  // The wave's rows of weights m0 + 16 rt + r16 of the outputs; with glu, its tiles alternate between gate and up rows.
  const int pair = a.glu ? 2 : 1, tile_rows = 16 * RT / pair, turn_rows = tiles * tile_rows;
  const int64_t wg_m0 = (int64_t)(blockIdx.x - slot * a.by_tiles.d) * ((int64_t)a.turns * turn_rows);
  if (expert == a.experts) {
    const uint32_t cols = a.turns * turn_rows;
    for (uint32_t i = threadIdx.x; i < 16 * cols; i += blockDim.x) {
      const uint32_t n = first + i / cols;
      const int64_t m = wg_m0 + i % cols;
      if (n < end && m < a.out_rows) store_y<DT>(a, n, m, 0.f);
    }
    return;
  }
  int turns = a.turns;  // of this workgroup: up to its last rows of weights
  while (turns > 1 && wg_m0 + (int64_t)(turns - 1) * turn_rows >= a.out_rows) --turns;
  int64_t m0 = wg_m0 + own * tile_rows;
  Few<C> f;
  f.split = a.split;
  auto start = [&](int64_t from) {  // the first unit of the tile at weight row `from`
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      int64_t m = from + 16 * (rt / pair) + r16;
      m = m < a.out_rows ? m : a.out_rows - 1;
      if (pair == 2 && (rt & 1)) m += a.out_rows;
      m += (int64_t)expert * a.M;
      f.codes[rt] = a.codes + m * a.row_bytes + part * (C::COLUMNS / 2) + quarter * 16;
      f.scales[rt] = a.scales + m * a.groups * (DT == 0 ? 4 : 2);
      f.zeros[rt] = a.zeros ? a.zeros + m * a.groups : a.codes;
    }
    f.unit = part;
  };
  const int rows = end - first < 16 ? end - first : 16;
  // All columns of x at once where they fit, or a unit or more for each of a tile's waves at a time.
  const bool fits = rows <= a.fit_rows;
  const int columns = fits ? a.all_columns : a.some_columns, pitch = 2 * columns + 16;
  const int whole = a.K / C::COLUMNS;
  const char* x = lds + (r16 < rows ? r16 : rows - 1) * pitch + quarter * 16;
  f32x4* sums = reinterpret_cast<f32x4*>(lds + a.x_bytes);
  const CodeBits<DT> bits;
  f32x4 sum[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) sum[rt] = f32x4{0, 0, 0, 0};
  Unit<C> even, odd;
  int turn = 0;

  auto times = [&](Unit<C>& o, int unit) { multiply(bits, o, x + unit * (2 * C::COLUMNS), rows * pitch, sum); };
  // A tile's end: its waves join their sums, and it is stored.  Lane (r16, quarter) has rows 4 quarter .. + 4 of x.
  auto finish = [&]() {
    if (a.split > 1) {
      f32x4* now = sums + (turn & 1) * (waves * RT * 64);  // the other half may still be read from
      if (part) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) now[(wave * RT + rt) * 64 + lane] = sum[rt];
      }
      __syncthreads();
      if (!part) {
        for (int w = wave + 1; w < wave + a.split; ++w)
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) sum[rt] += now[(w * RT + rt) * 64 + lane];
      }
    }
    if (!part) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        if (pair == 2 && (rt & 1)) continue;
        const int64_t m = m0 + 16 * (rt / pair) + r16;
        if (m >= a.out_rows) continue;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t n = first + 4 * quarter + k;
          if (n < end) store_y<DT>(a, n, m, pair == 2 ? silu(sum[rt][k]) * sum[rt + 1 < RT ? rt + 1 : rt][k] : sum[rt][k]);
        }
      }
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) sum[rt] = f32x4{0, 0, 0, 0};
    ++turn;
    m0 += turn_rows;
  };

  if (fits && whole * C::COLUMNS == a.K && part < whole) {
    // Whole units, two in turn through all turns: each is loaded while the other one is worked on.
    start(m0);
    load_weights<false>(a, f, even);
    stage_x<DT>(a, first, rows, 0, a.by_all, pitch, lds);
    __syncthreads();
    bool more, ends;
    int now;
    auto next = [&]() {
      now = f.unit;
      f.advance();
      ends = f.unit >= whole;
      more = !ends || turn + 1 < turns;
      if (ends && more) start(m0 + turn_rows);
    };
    for (;;) {
      next();
      if (!more) {
        times(even, now);
        break;
      }
      load_weights<false>(a, f, odd);
      times(even, now);
      if (ends) finish();
      next();
      if (!more) {
        times(odd, now);
        break;
      }
      load_weights<false>(a, f, even);
      times(odd, now);
      if (ends) finish();
    }
    finish();
    return;
  }
  // K that ends inside a unit, or more of x than fits.
  for (int t = 0; t < turns; ++t) {
    start(m0);
    for (int k0 = 0; k0 < a.K; k0 += columns) {
      const int first_unit = k0 / C::COLUMNS, end_unit = first_unit + columns / C::COLUMNS;
      const int last = end_unit < whole ? end_unit : whole;
      if (f.unit < last) load_weights<false>(a, f, even);
      if (t == 0 || !fits) {
        if (t || k0) __syncthreads();
        stage_x<DT>(a, first, rows, k0, fits ? a.by_all : a.by_some, pitch, lds);
        __syncthreads();
      }
      if (f.unit < last) {
        for (;;) {
          int now = f.unit;
          f.advance();
          if (f.unit >= last) {
            times(even, now - first_unit);
            break;
          }
          load_weights<false>(a, f, odd);
          times(even, now - first_unit);
          now = f.unit;
          f.advance();
          if (f.unit >= last) {
            times(odd, now - first_unit);
            break;
          }
          load_weights<false>(a, f, even);
          times(odd, now - first_unit);
        }
      }
      if (f.unit == whole && whole * C::COLUMNS < a.K && whole < end_unit) {
        load_weights<true>(a, f, even);
        times(even, whole - first_unit);
      }
    }
    finish();
  }
}

// ------------------------------------------------------------------- to 4 bits

struct QuantArgs {
  const char* w;
  uint8_t* codes;
  char* scales;
  uint8_t* zeros;
  int64_t rows;  // of all matrices
  int64_t row_bytes;
  int32_t K, group, groups;
};

// A wave has a group of a row.
template <int DT>
__global__ __launch_bounds__(256) void q4_quantize_kernel(const QuantArgs a) {
  typedef Type<DT> T;
  const int lane = threadIdx.x & 63;
  const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (at >= a.rows * a.groups) return;
  const int64_t row = at / a.groups;
  const int k0 = (int)(at - row * a.groups) * a.group, k1 = a.K - k0 < a.group ? a.K : k0 + a.group;
  const typename T::elt* w = reinterpret_cast<const typename T::elt*>(a.w) + row * a.K;
  float lo = 0.f, hi = 0.f;
  for (int k = k0 + lane; k < k1; k += 64) {
    const float v = T::widen(w[k]);
    lo = fminf(lo, v);
    hi = fmaxf(hi, v);
  }
  for (int d = 32; d; d /= 2) {
    lo = fminf(lo, __shfl_xor(lo, d));
    hi = fmaxf(hi, __shfl_xor(hi, d));
  }
  const typename T::elt scale = T::narrow(a.zeros ? (hi - lo) / 15.f : fmaxf(hi, -lo) / 7.f);
  const float s = T::widen(scale);
  float zero = 8.f;
  if (a.zeros) zero = s > 0.f ? fminf(fmaxf(rintf(-lo / s), 0.f), 15.f) : 0.f;
  if (lane == 0) {
    reinterpret_cast<typename T::elt*>(a.scales)[at] = scale;
    if (a.zeros) a.zeros[at] = (uint8_t)zero;
  }
  uint8_t* out = a.codes + row * a.row_bytes;
  for (int k = k0 + 2 * lane; k < k1; k += 128) {  // a byte: groups begin at even columns
    uint32_t byte = 0;
    for (int i = 0; i < 2 && k + i < k1; ++i) {
      const float q = s > 0.f ? rintf(T::widen(w[k + i]) / s) + zero : zero;
      byte |= (uint32_t)fminf(fmaxf(q, 0.f), 15.f) << (4 * i);
    }
    out[k / 2] = (uint8_t)byte;
  }
}

typedef void (*q4_fn)(const Q4Args);

template <int DT, int RT>
q4_fn pick_shape(bool whole, bool zeros) {
  return whole ? (zeros ? q4_few_kernel<FewShape<DT, RT, true, true>> : q4_few_kernel<FewShape<DT, RT, true, false>>)
               : (zeros ? q4_few_kernel<FewShape<DT, RT, false, true>> : q4_few_kernel<FewShape<DT, RT, false, false>>);
}

template <int RT>
q4_fn pick_few(int dt, bool whole, bool zeros) {
  return dt == EBAG_F32 ? pick_shape<0, RT>(whole, zeros) : dt == EBAG_F16 ? pick_shape<1, RT>(whole, zeros) : pick_shape<2, RT>(whole, zeros);
}

int hipf(hipError_t e, const char* what) { return fail(EBAG_EHIP, "%s: %s", what, hipGetErrorString(e)); }

}  // namespace

struct gemv_ar_q4_plan {
  int device = 0;
  int64_t M = 0, K = 0;
  int32_t group = 0, dtype = 0, experts = 0, glu = 0;
};

namespace {

int check_plan(const gemv_ar_q4_plan* h) {
  if (!h) return fail(EBAG_EINVAL, "null plan");
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev != h->device)
    return fail(EBAG_EINVAL, "the plan belongs to device %d, but device %d is current", h->device, dev);
  return EBAG_OK;
}

int elt_of(int dtype) { return dtype == EBAG_F32 ? 4 : 2; }

int fill_args(const gemv_ar_q4_plan* h, const uint8_t* codes, const void* scales, const uint8_t* zeros, const void* x,
              int64_t ldx, int64_t x_rows, int64_t rows, void* y, int64_t ldy, int32_t y_dtype, Q4Args* a) {
  if (y_dtype != h->dtype && y_dtype != EBAG_F32)
    return fail(EBAG_EINVAL, "y_dtype must be fp32 or the plan's type, not %d", (int)y_dtype);
  if (!codes || !scales || !x || !y) return fail(EBAG_EINVAL, "null codes, scales, x or y");
  const int elt = elt_of(h->dtype), y_elt = elt_of(y_dtype);
  const int64_t wide = h->glu ? h->M / 2 : h->M;
  if (reinterpret_cast<uintptr_t>(scales) % elt || reinterpret_cast<uintptr_t>(x) % elt ||
      reinterpret_cast<uintptr_t>(y) % y_elt)
    return fail(EBAG_EINVAL, "scales, x or y not aligned to its elements");
  if (ldx < h->K || ldx > (int64_t)1 << 40) return fail(EBAG_EINVAL, "row step %lld of x below K=%lld", (long long)ldx, (long long)h->K);
  if (ldy < wide || ldy > (int64_t)1 << 40) return fail(EBAG_EINVAL, "row step %lld of y below its %lld columns", (long long)ldy, (long long)wide);
  *a = Q4Args{};
  a->codes = codes;
  a->scales = static_cast<const char*>(scales);
  a->zeros = zeros;
  a->x = static_cast<const char*>(x);
  a->y = static_cast<char*>(y);
  a->ldx = ldx * elt;
  a->ldy = ldy * y_elt;
  a->row_bytes = (h->K + 1) / 2;
  a->codes_bytes = a->row_bytes * h->M * h->experts;
  a->M = h->M;
  a->out_rows = wide;
  a->x_rows = x_rows;
  a->rows = (uint32_t)rows;
  a->K = (int32_t)h->K;
  a->group = h->group;
  a->groups = (int32_t)((h->K + h->group - 1) / h->group);
  a->experts = h->experts;
  a->glu = h->glu;
  a->y_f32 = y_dtype == EBAG_F32;
  a->by_choices = make_divisor(1);
  a->by_group_blocks = make_divisor(h->group / 32);
  return EBAG_OK;
}

// Most tiles of `cols` rows that `rows` rows of `experts` experts and the
// dropped rows behind them can make.
int64_t most_tiles(int64_t rows, int64_t experts, int64_t cols) {
  const int64_t n = (rows + (experts + 1) * (cols - 1)) / cols;
  return n < rows ? n : rows;
}

int launch_few(const gemv_ar_q4_plan* h, Q4Args a, hipStream_t stream) {
  const int rt = h->glu ? 2 : 1, parts = h->dtype == EBAG_F32 ? 3 : 1;
  const bool whole = h->group % 128 == 0;
  const int columns = whole ? 512 : 256;
  const int units = (a.K + columns - 1) / columns;
  const int rows = a.rows < 16 ? (int)a.rows : 16;
  const int64_t slots = a.offsets ? most_tiles(a.rows, h->experts, 16) : (a.rows + 15) / 16;
  const int64_t all_tiles = (a.out_rows + 15) / 16 * slots;
  // A tile's waves: 2048 in all, and with few rows 1024 bytes of a weight row at a time.  x is staged once for a
  // workgroup's tiles, so with more rows of x fewer waves to a tile are better where there are tiles enough (20000 x 4096
  // with 8 rows: four waves to a tile 20.8 us, two 16.8), and more where there are not (4096 x 4096 with 16 rows: four
  // 10.7, eight 7.9; with one row 5.4 and 5.8).
  const bool many = rows >= 4 || units >= 16;
  const int waves = many && all_tiles * 4 < 2048 && units >= 8 ? 8 : 4;
  // LDS: x and the waves' sums, two of each tile's; three workgroups on a CU, or one where there are no more of them
  // than CUs.
  const int sums = 2 * waves * rt * 64 * (int)sizeof(f32x4), most = waves == 8 ? kCuLds - sums : 49152;
  auto fits = [&](int split) { return rows * parts * (2 * split * columns + 16) + 16 <= most; };
  a.split = 1;
  while (a.split < waves && a.split * 2 <= units && fits(a.split * 2) &&
         (all_tiles * a.split < 2048 || (rows < 4 && a.row_bytes > 1024 * a.split)))
    a.split *= 2;
  // Its turns: about 2048 workgroups, or 1024 of twice the weights (128 experts of 2 x 1024 x 2048, two rows each: 66
  // us with 2048, 63.5 with 1024, 60 with 512; 64 experts of 4096 x 2048, four rows each: 59, 66 and 102 us).
  const int64_t turn_rows = 16 * (waves / a.split);
  const int64_t all_turns = (a.out_rows + turn_rows - 1) / turn_rows;
  int64_t turns = all_turns * slots / (rt == 2 ? 1024 : 2048);
  turns = turns < 1 ? 1 : turns > all_turns ? all_turns : turns;
  a.turns = (int)turns;
  const int64_t tiles = (all_turns + turns - 1) / turns;
  if (tiles * slots > INT_MAX) return fail(EBAG_EUNSUPPORTED, "too many tiles for one launch");
  a.by_tiles = make_divisor(tiles);
  // LDS for x: 40 KiB, or a turn's columns of 16 rows where they are more.
  const int64_t least = (int64_t)rows * parts * (2 * a.split * columns + 16);
  const int64_t room = least > 40960 ? least : 40960;
  a.all_columns = units * columns;
  const int64_t fit = room / (parts * (2 * (int64_t)a.all_columns + 16));
  a.fit_rows = fit < rows ? (int)fit : rows;
  a.some_columns = (int)((room / (rows * parts) - 16) / (2 * a.split * columns)) * a.split * columns;
  a.by_all = make_divisor(a.all_columns / 8);
  a.by_some = make_divisor(a.some_columns / 8);
  a.x_bytes = (int)(a.fit_rows < rows ? (room + 15) / 16 * 16 : rows * parts * (2 * (int64_t)a.all_columns + 16));
  const size_t lds = a.x_bytes + (a.split > 1 ? sums : 0);
  const q4_fn fn = rt == 1 ? pick_few<1>(h->dtype, whole, a.zeros) : pick_few<2>(h->dtype, whole, a.zeros);
  hipLaunchKernelGGL(fn, dim3((unsigned)(tiles * slots)), dim3(64 * waves), lds, stream, a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? EBAG_OK : hipf(e, "launch the product with 4-bit weights");
}

int launch_tile(const gemv_ar_q4_plan* h, Q4Args a, int x_tiles, hipStream_t stream) {
  const int64_t cols = 32 * x_tiles, per_wg = kQ4TileRows / (h->glu ? 2 : 1);
  const int64_t tiles = (a.out_rows + per_wg - 1) / per_wg;
  const int64_t slots = a.offsets ? most_tiles(a.rows, h->experts, cols) : (a.rows + cols - 1) / cols;
  if (tiles * slots > INT_MAX) return fail(EBAG_EUNSUPPORTED, "too many tiles for one launch");
  a.by_tiles = make_divisor(tiles);
  launch_q4_tile(a, h->dtype, x_tiles, (unsigned)(tiles * slots), stream);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? EBAG_OK : hipf(e, "launch the product with 4-bit weights");
}

// Which kernel: the one with the least time by what was measured at K = 4096 (all
// grow with K alike): the kernel for few rows takes 8.0 ns for every 16 x 16 tile of
// weight rows and rows of x; the matrix-product kernel with 32 rows of x 157 ns for
// a workgroup, with 64 203 ns, and never less than 45 and 62 us, a workgroup's own
// time.  Where a step of 128 columns has several scales: 12.5 ns, and with 64 rows 480
// ns and 107 us.  (64 experts of 4096 x 2048, in us by the three: 12 rows each 94, 89, 101; 48
// rows 280, 141, 129.  One matrix of 8192 x 4096: 64 rows 22, 48, 67; 256 rows 64, 49,
// 67.)  An expert's rows fill their last tile half on average.
int launch(const gemv_ar_q4_plan* h, const Q4Args& a, hipStream_t stream) {
  if (h->dtype == EBAG_F32 || h->K >= 1 << 27) return launch_few(h, a, stream);
  const bool whole = h->group % 128 == 0;
  auto tiles = [&](double rows, double cols) {  // of `rows` weight rows and `cols` rows of x
    const double experts = a.offsets ? h->experts : 1, some = a.rows < experts ? a.rows : experts;
    const double slots = a.offsets ? a.rows / cols + experts / 2 : 0, all = (a.rows + (int)cols - 1) / (int)cols;
    const double n = a.offsets ? (slots < some ? some : slots) : all;
    return (double)((h->M + (int)rows - 1) / (int)rows) * (n < a.rows ? n : a.rows);
  };
  auto at_least = [](double v, double least) { return v < least ? least : v; };
  const double few = tiles(16, 16) * (whole ? 0.0080 : 0.0125);
  const double one = at_least(tiles(kQ4TileRows, 32) * 0.157, 45);
  const double two = at_least(tiles(kQ4TileRows, 64) * (whole ? 0.203 : 0.48), whole ? 62 : 107);
  if (few <= two && (few <= one || !whole)) return launch_few(h, a, stream);
  return launch_tile(h, a, whole && one <= two ? 1 : 2, stream);
}

}  // namespace

extern "C" {

int gemv_ar_q4_create(gemv_ar_q4_t* out, int64_t M, int64_t K, int32_t group, int32_t dtype, int32_t experts,
                      int32_t glu) {
  if (!out) return fail(EBAG_EINVAL, "null output handle");
  *out = nullptr;
  if (M < 1 || M > INT_MAX) return fail(EBAG_EINVAL, "M=%lld outside [1, 2^31)", (long long)M);
  if (K < 1 || K > INT_MAX - 4096) return fail(EBAG_EINVAL, "K=%lld outside [1, 2^31 - 4096)", (long long)K);
  if (M > ((int64_t)1 << 40) / K) return fail(EBAG_EINVAL, "M * K above 2^40");
  if (group < 32 || group % 32) return fail(EBAG_EINVAL, "group=%d is not a positive multiple of 32", group);
  if (dtype != EBAG_F32 && dtype != EBAG_F16 && dtype != EBAG_BF16) return fail(EBAG_EINVAL, "bad dtype %d", (int)dtype);
  if (experts < 1 || experts > 512) return fail(EBAG_EINVAL, "experts=%d outside [1, 512]", experts);
  if (glu != 0 && glu != 1) return fail(EBAG_EINVAL, "glu must be 0 or 1");
  if (glu && M % 2) return fail(EBAG_EINVAL, "glu needs an even M, not %lld", (long long)M);
  gemv_ar_q4_plan* h = new (std::nothrow) gemv_ar_q4_plan();
  if (!h) return fail(EBAG_ENOMEM, "host allocation failed");
  const hipError_t e = hipGetDevice(&h->device);
  if (e != hipSuccess) {
    delete h;
    return hipf(e, "query device");
  }
  h->M = M;
  h->K = K;
  h->group = group;
  h->dtype = dtype;
  h->experts = experts;
  h->glu = glu;
  *out = h;
  clear_error();
  return EBAG_OK;
}

int gemv_ar_q4_quantize(gemv_ar_q4_t h, const void* w, uint8_t* codes, void* scales, uint8_t* zeros,
                        hipStream_t stream) {
  if (int rc = check_plan(h)) return rc;
  if (!w || !codes || !scales) return fail(EBAG_EINVAL, "null w, codes or scales");
  const int elt = elt_of(h->dtype);
  if (reinterpret_cast<uintptr_t>(w) % elt || reinterpret_cast<uintptr_t>(scales) % elt)
    return fail(EBAG_EINVAL, "w or scales not aligned to its elements");
  QuantArgs a{};
  a.w = static_cast<const char*>(w);
  a.codes = codes;
  a.scales = static_cast<char*>(scales);
  a.zeros = zeros;
  a.rows = h->M * h->experts;
  a.row_bytes = (h->K + 1) / 2;
  a.K = (int32_t)h->K;
  a.group = h->group;
  a.groups = (int32_t)((h->K + h->group - 1) / h->group);
  const int64_t wgs = (a.rows * a.groups + 3) / 4;
  if (wgs > INT_MAX) return fail(EBAG_EUNSUPPORTED, "too many groups for one launch");
  void (*fn)(const QuantArgs) = h->dtype == EBAG_F32   ? q4_quantize_kernel<0>
                                : h->dtype == EBAG_F16 ? q4_quantize_kernel<1>
                                                       : q4_quantize_kernel<2>;
  hipLaunchKernelGGL(fn, dim3((unsigned)wgs), dim3(256), 0, stream, a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? EBAG_OK : hipf(e, "launch the rounding to 4 bits");
}

int gemv_ar_q4_forward(gemv_ar_q4_t h, const uint8_t* codes, const void* scales, const uint8_t* zeros, const void* x,
                       int64_t ldx, int64_t rows, void* y, int64_t ldy, int32_t y_dtype, hipStream_t stream) {
  if (int rc = check_plan(h)) return rc;
  if (rows < 0 || rows > INT_MAX) return fail(EBAG_EINVAL, "rows=%lld outside [0, 2^31)", (long long)rows);
  if (!rows) return EBAG_OK;
  Q4Args a;
  if (int rc = fill_args(h, codes, scales, zeros, x, ldx, rows, rows, y, ldy, y_dtype, &a)) return rc;
  return launch(h, a, stream);
}

int gemv_ar_q4_experts(gemv_ar_q4_t h, const uint8_t* codes, const void* scales, const uint8_t* zeros, const void* x,
                       int64_t ldx, int64_t x_rows, const int32_t* offsets, const int32_t* src, int32_t choices,
                       int64_t rows, void* y, int64_t ldy, int32_t y_dtype, hipStream_t stream) {
  if (int rc = check_plan(h)) return rc;
  if (rows < 0 || rows > INT_MAX) return fail(EBAG_EINVAL, "rows=%lld outside [0, 2^31)", (long long)rows);
  if (!rows) return EBAG_OK;
  if (!offsets) return fail(EBAG_EINVAL, "null offsets");
  if (src && choices < 1) return fail(EBAG_EINVAL, "choices=%d must be positive", choices);
  if (x_rows < 1 || x_rows > INT_MAX || (!src && x_rows != rows))
    return fail(EBAG_EINVAL, "x_rows=%lld: without src x has as many rows as y", (long long)x_rows);
  Q4Args a;
  if (int rc = fill_args(h, codes, scales, zeros, x, ldx, x_rows, rows, y, ldy, y_dtype, &a)) return rc;
  a.offsets = offsets;
  a.src = src;
  a.by_choices = make_divisor(src ? choices : 1);
  return launch(h, a, stream);
}

void gemv_ar_q4_destroy(gemv_ar_q4_t h) { delete h; }

}  // extern "C"
