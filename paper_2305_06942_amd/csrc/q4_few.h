// The kernel with 4-bit weights for few rows of x, instantiated for one storage
// type of x by each q4_few_*.hip.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "lanes.h"
#include "q4.h"

namespace ebag {
namespace {

// A tile is 16 rows of weights (RT = 2 with glu: 16 gate rows and the up rows that go
// with them) and up to 16 rows of x; `split` waves share one, each taking every
// split-th unit of 512 or 256 columns (256 or 128 bytes of codes), and join their sums
// in LDS at the end.  A workgroup has 4 or 8 waves on one tile or several and goes on
// to the tiles of `turns` more rows of weights with the same x in LDS.  A lane loads
// 16 bytes, 32 consecutive codes of row lane % 16; a transposition between the four
// lanes of a row (lane / 16) then gives word t of each the columns 32 t + 8 (lane / 16)
// .. + 8, the layout of a 16x16x32 matrix instruction over 32 consecutive columns,
// which belong to one group.  x is the first operand, so a lane holds sums of ONE
// weight row for four rows of x and needs one scale per group: the four lanes of a row
// load those of four blocks of 32 columns (or of four steps, where a group is several
// blocks) and pass them round.  Rows of a tile beyond the last one repeat it; nothing
// they give is stored.
//
// The loads of a wave's next unit are under way while it works on one.
//
// Bound by the codes' bytes with one to four rows: 65536 x 8192 fp16, one row, 277 MB
// in 56 us, 4.9 TB/s (this pattern of 16 rows a wave reads 5.3 to 5.5 and a plain
// stream 6.5); 128 experts of 2 x 1024 x 2048, two rows each, 246 MB in 57 us.  A launch
// of a few MB is bound by its chain of launch, x, codes, join and store: 4096 x 4096,
// one row, 5.5 us.  Many rows of x, or scales for every 32 columns, bound it by the
// latency of a unit's small steps and by staging x: 12 x 10001 x 5001 26 us, 60 experts
// of 1400 x 1000 with 20 rows each 30 us, 22 with groups of 128.

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

constexpr int kFewThreads = 512;

// What a launch is compiled for.  WHOLE: a group is a multiple of 128 columns, so
// a step of 128 has one scale.  ZEROS: there are zero points.  Y32: y is fp32.  WORDS: rows of codes
// begin at multiples of 4 bytes.  Others are loaded from the multiple of 4 below and
// shifted in registers: memory takes 16 bytes at any address, but not as fast (1 x
// 40000 x 5110, rows of 2555 bytes: 43.9 us; rows of 2556: 28.7 us; shifted 32.7 us).
template <int DT_, int RT_, bool WHOLE_, bool ZEROS_, bool WORDS_, bool Y32_>
struct FewShape {
  static constexpr int DT = DT_, RT = RT_;
  static constexpr bool WHOLE = WHOLE_, ZEROS = ZEROS_, WORDS = WORDS_, Y32 = Y32_;
  static constexpr int STEPS = WHOLE ? 4 : 2;     // of a unit
  static constexpr int SCALES = WHOLE ? 1 : STEPS;  // loads of scales of a unit: four lanes of a row load one each
  static constexpr int COLUMNS = 128 * STEPS;
};

// Where a lane of a wave with RT tiles of weight rows loads its next unit from.
template <class C>
struct Few {
  const uint8_t* codes[C::RT];  // its row of weights, its quarter's bytes (from the multiple of 4 below on)
  const char* scales[C::RT];    // that row's first scale
  const uint8_t* zeros[C::RT];  // and zero
  int behind[C::RT];            // not WORDS: how far on the word behind the row's last one in a unit is
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
  uint32_t behind[C::RT];  // not WORDS: the word behind the row's last one here
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
      o.w[s][rt] = !END ? load16(reinterpret_cast<const char*>(p)) : C::WORDS ? load_codes_end(a, p) : load_words_end(a, p);
    }
  if (!C::WORDS) {
#pragma unroll
    for (int rt = 0; rt < C::RT; ++rt) {
      const uint8_t* p = f.codes[rt] + f.behind[rt];
      if (END && p >= a.codes + a.codes_bytes) p = f.codes[rt] - 16 * quarter;  // not used: any word of the row
      o.behind[rt] = *reinterpret_cast<const uint32_t*>(p);
    }
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
// shift: not WORDS: how many bytes a row begins behind a multiple of 4.
template <class C>
__device__ __forceinline__ void multiply(const CodeBits<C::DT, C::Y32>& bits, Unit<C>& o, const char* x, int pitch,
                                         const uint32_t* shift, f32x4* sum) {
  typedef Q4Type<C::DT> Q;
  typedef Type<C::DT> T;
  constexpr int PARTS = Q::PARTS, RT = C::RT;
  constexpr bool F32 = C::DT == 0;
  const vec16 ones = {Q::ONES, Q::ONES, Q::ONES, Q::ONES};
  uint32_t all[RT][4], zero[RT][4];  // scale, and the zero above it or in a word of its own
  if (!C::WORDS) {
    // A lane's next word is the first one of the row's next quarter, 16 lanes on; the last quarter's is in the next step.
    const int lane = threadIdx.x & 63, on = (lane + 16 & 63) * 4;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      uint32_t first[C::STEPS + 1];
#pragma unroll
      for (int s = 0; s < C::STEPS; ++s) first[s] = __builtin_amdgcn_ds_bpermute(on, o.w[s][rt][0]);
      first[C::STEPS] = o.behind[rt];
#pragma unroll
      for (int s = 0; s < C::STEPS; ++s) {
        vec16& w = o.w[s][rt];
        const uint32_t next = lane < 48 ? first[s] : first[s + 1];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = __builtin_amdgcn_alignbyte(j < 3 ? w[j < 3 ? j + 1 : 3] : next, w[j], shift[rt]);
      }
    }
  }
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
      if (!C::Y32) xsum = Q::mfma(xs[0], ones, C::WHOLE && t ? xsum : f32x4{0, 0, 0, 0});
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const int g = C::WHOLE ? 0 : t;
        vec16 q = unpack_codes(bits, o.w[s][rt][t]);
        if constexpr (C::Y32) q = centred(bits, q, off[rt][g]);
        if (!C::WHOLE || t == 0) v[rt] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int p = 0; p < PARTS; ++p) v[rt] = Q::mfma(xs[p], q, v[rt]);
        if (C::WHOLE && t < 3) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          sum[rt][i] = __builtin_fmaf(scale[rt][g], C::Y32 ? v[rt][i] : __builtin_fmaf(off[rt][g], xsum[i], v[rt][i]), sum[rt][i]);
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
      const int on = 8 * (int)c;  // k0 + on may pass 2^31, K - k0 is positive
      load_x<DT>(a.x + row * a.ldx + ((int64_t)k0 + on) * ELT, a.K - k0 - on, a.K, v[j]);
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
__global__ __launch_bounds__(kFewThreads, C::RT == 2 ? 2 : C::DT == 0 ? 3 : 4) void q4_few_kernel(const Q4Args a) {
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
      if (n < end && m < a.out_rows) store_y<DT, C::Y32>(a, n, m, 0.f);
    }
    return;
  }
  int turns = a.turns;  // of this workgroup: up to its last rows of weights
  while (turns > 1 && wg_m0 + (int64_t)(turns - 1) * turn_rows >= a.out_rows) --turns;
  int64_t m0 = wg_m0 + own * tile_rows;
  Few<C> f;
  f.split = a.split;
  // Rows of one lane in different turns are a multiple of 16 rows apart, so they begin equally far behind a multiple of 4
  // (but for those that stand in for rows behind the last, whose results are not used).
  uint32_t shift[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int64_t m = m0 + 16 * (rt / pair) + r16 + (pair == 2 && (rt & 1) ? a.out_rows : 0) + (int64_t)expert * a.M;
    shift[rt] = C::WORDS ? 0 : (uint32_t)(reinterpret_cast<uintptr_t>(a.codes + m * a.row_bytes) & 3);
  }
  auto start = [&](int64_t from) {  // the first unit of the tile at weight row `from`
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      int64_t m = from + 16 * (rt / pair) + r16;
      m = m < a.out_rows ? m : a.out_rows - 1;
      if (pair == 2 && (rt & 1)) m += a.out_rows;
      m += (int64_t)expert * a.M;
      f.codes[rt] = a.codes + m * a.row_bytes + part * (C::COLUMNS / 2) + quarter * 16;
      if (!C::WORDS) {
        const int off = (int)(reinterpret_cast<uintptr_t>(f.codes[rt]) & 3);
        f.codes[rt] -= off;
        f.behind[rt] = C::STEPS * 64 - 16 * quarter - (off ? 0 : 4);  // a row on a multiple of 4 needs no word behind
      }
      f.scales[rt] = a.scales + m * a.groups * (DT == 0 ? 4 : 2);
      f.zeros[rt] = a.zeros ? a.zeros + m * a.groups : a.codes;
    }
    f.unit = part;
  };
  const int rows = end - first < 16 ? end - first : 16;
  // All columns of x at once where they fit, or a unit or more for each of a tile's waves at a time.
  const bool fits = rows <= a.fit_rows;
  const int columns = fits ? a.all_columns : a.some_columns, pitch = 2 * columns + 16;
  const int whole = a.K / C::COLUMNS, units = (a.K + C::COLUMNS - 1) / C::COLUMNS;
  const char* x = lds + (r16 < rows ? r16 : rows - 1) * pitch + quarter * 16;
  f32x4* sums = reinterpret_cast<f32x4*>(lds + a.x_bytes);
  const CodeBits<DT, C::Y32> bits;
  f32x4 sum[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) sum[rt] = f32x4{0, 0, 0, 0};
  Unit<C> even, odd;
  int turn = 0;

  auto times = [&](Unit<C>& o, int unit) { multiply(bits, o, x + unit * (2 * C::COLUMNS), rows * pitch, shift, sum); };
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
          if (n < end) store_y<DT, C::Y32>(a, n, m, pair == 2 ? silu<C::Y32>(sum[rt][k]) * sum[rt + 1 < RT ? rt + 1 : rt][k] : sum[rt][k]);
        }
      }
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) sum[rt] = f32x4{0, 0, 0, 0};
    ++turn;
    m0 += turn_rows;
  };

  auto load = [&](Unit<C>& o) {
    if (f.unit < whole)
      load_weights<false>(a, f, o);
    else
      load_weights<true>(a, f, o);
  };

  // x: all columns once, or the part that has a unit, for every tile anew.  All of a tile's waves come here as often.
  int from_unit = 0, to_unit = 0;
  auto stage = [&]() {
    from_unit = to_unit;
    to_unit = fits ? units : from_unit + columns / C::COLUMNS;
    __syncthreads();
    stage_x<DT>(a, first, rows, from_unit * C::COLUMNS, fits ? a.by_all : a.by_some, pitch, lds);
    __syncthreads();
  };
  // Two units in turn through all turns: each is loaded while the other one is worked on.
  start(m0);
  load(even);
  bool more, ends;
  int now;
  auto next = [&]() {
    now = f.unit;
    if (now >= to_unit) stage();
    f.advance();
    ends = f.unit >= units;
    more = !ends || turn + 1 < turns;
    if (ends && more) start(m0 + turn_rows);
  };
  auto end_tile = [&]() {
    if (!fits) {
      while (to_unit < units) stage();
      to_unit = 0;
    }
    finish();
  };
  for (;;) {
    next();
    if (!more) {
      times(even, now - from_unit);
      break;
    }
    load(odd);
    times(even, now - from_unit);
    if (ends) end_tile();
    next();
    if (!more) {
      times(odd, now - from_unit);
      break;
    }
    load(even);
    times(odd, now - from_unit);
    if (ends) end_tile();
  }
  end_tile();
}

// The instance for a launch.
template <int DT>
q4_fn pick_few(const Q4FewKind& k) {
  auto codes = [&](auto rt, auto whole, auto y32) -> q4_fn {
    constexpr int RT = decltype(rt)::value;
    constexpr bool WHOLE = decltype(whole)::value, Y32 = decltype(y32)::value;
    if (k.words)
      return k.zeros ? q4_few_kernel<FewShape<DT, RT, WHOLE, true, true, Y32>> : q4_few_kernel<FewShape<DT, RT, WHOLE, false, true, Y32>>;
    return k.zeros ? q4_few_kernel<FewShape<DT, RT, WHOLE, true, false, Y32>> : q4_few_kernel<FewShape<DT, RT, WHOLE, false, false, Y32>>;
  };
  auto result = [&](auto rt, auto whole) -> q4_fn {
    if constexpr (DT != 0)
      if (!k.y32) return codes(rt, whole, std::false_type());
    return codes(rt, whole, std::true_type());
  };
  const std::integral_constant<int, 1> one;
  const std::integral_constant<int, 2> two;
  if (k.tiles == 1) return k.whole ? result(one, std::true_type()) : result(one, std::false_type());
  return k.whole ? result(two, std::true_type()) : result(two, std::false_type());
}

}  // namespace
}  // namespace ebag
