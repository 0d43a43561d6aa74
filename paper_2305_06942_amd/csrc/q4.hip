// Products with 4-bit weights (gemv_ar_q4_* of include/gemv_ar.h): rounding to 4
// bits, and the kernel for few rows of x.
#include <hip/hip_runtime.h>

#include <climits>
#include <new>

#include "ebag_a2a.h"
#include "gemv_ar.h"
#include "q4.h"

using namespace ebag;

namespace {

// ------------------------------------------------------------------- few rows
//
// A workgroup has RT tiles of 16 rows of weights and CT tiles of 16 rows of x;
// its waves split K in units of 256 columns (a cache line of codes), wave w
// taking units w, w + waves, ..., and join their sums in LDS at the end.  A
// lane loads 16 bytes, 32 consecutive codes of row lane % 16; a transposition
// between the four lanes of a row (lane / 16) then gives word t of each the
// columns 32 t + 8 (lane / 16) .. + 8, the layout of a 16x16x32 matrix
// instruction over 32 consecutive columns, which belong to one group.  x is
// the first operand, so a lane holds sums of ONE weight row for four rows of x
// and needs one scale per group.  Rows of a tile beyond the last one repeat it;
// nothing they give is stored.

constexpr int kUnit = 2;  // steps of 128 columns

__device__ __forceinline__ void transpose_words(vec16& w) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
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

// 16 bytes of codes at `byte` of a row; what lies behind the row's end is not
// used, what lies behind the last matrix is not read.
__device__ __forceinline__ vec16 load_codes(const Q4Args& a, const uint8_t* row, int64_t byte) {
  const uint8_t* p = row + byte;
  if (p + 16 <= a.codes + a.codes_bytes) return load16(reinterpret_cast<const char*>(p));
  vec16 r = {0, 0, 0, 0};
  for (int i = 0; i < 16; ++i)
    if (p + i < a.codes + a.codes_bytes) r[i / 4] |= (uint32_t)p[i] << (8 * (i % 4));
  return r;
}

// Eight elements of x from column k on, in pair order.  TAIL: with zeros behind
// column K.
template <int DT, bool TAIL>
__device__ __forceinline__ void load_x(const char* row, int k, int K, vec16* parts) {
  constexpr int ELT = DT == 0 ? 4 : 2, VECS = DT == 0 ? 2 : 1;
  vec16 v[VECS];
  if (TAIL) {
#pragma unroll
    for (int i = 0; i < VECS; ++i) v[i] = vec16{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (k + i >= K) continue;
      if (DT == 0)
        v[i / 4][i % 4] = reinterpret_cast<const uint32_t*>(row)[k + i];
      else
        v[0][i / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(row)[k + i] << (16 * (i % 2));
    }
  } else {
#pragma unroll
    for (int i = 0; i < VECS; ++i) v[i] = load16(row + (int64_t)k * ELT + 16 * i);
  }
  if (DT == 0)
    split_f32(v[0], v[VECS - 1], parts);
  else
    parts[0] = pair_order(v[0]);
}

// What a lane of a wave with RT x CT tiles works on.
template <int RT, int CT>
struct Few {
  const uint8_t* codes[RT];  // its row of weights
  int64_t groups[RT];        // that row's first scale
  const char* x[CT];         // its row of x
  f32x4 sum[RT][CT];
};

// 128 columns: w holds the lane's codes.
template <int DT, int RT, int CT, bool TAIL>
__device__ __forceinline__ void few_step(const Q4Args& a, Few<RT, CT>& f, vec16* w, int step) {
  typedef Q4Type<DT> Q;
  typedef Type<DT> T;
  constexpr int PARTS = Q::PARTS;
  const vec16 ones = {Q::ONES, Q::ONES, Q::ONES, Q::ONES};
  const int quarter = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) transpose_words(w[rt]);
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    int g = (int)divide_by(a.by_group_blocks, (uint32_t)(step * 4 + t));
    if (TAIL) g = g < a.groups ? g : a.groups - 1;
    vec16 xs[CT][PARTS];
    f32x4 xsum[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      load_x<DT, TAIL>(f.x[ct], step * 128 + 32 * t + 8 * quarter, a.K, xs[ct]);
      xsum[ct] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int p = 0; p < PARTS; ++p) xsum[ct] = Q::mfma(xs[ct][p], ones, xsum[ct]);
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const vec16 q = unpack_codes<DT>(w[rt][t]);
      const float scale = T::widen(reinterpret_cast<const typename T::elt*>(a.scales)[f.groups[rt] + g]);
      const float off = -16.f - (a.zeros ? (float)a.zeros[f.groups[rt] + g] : 8.f);
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        f32x4 v = {0, 0, 0, 0};
#pragma unroll
        for (int p = 0; p < PARTS; ++p) v = Q::mfma(xs[ct][p], q, v);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          f.sum[rt][ct][i] = __builtin_fmaf(scale, __builtin_fmaf(off, xsum[ct][i], v[i]), f.sum[rt][ct][i]);
      }
    }
    if (TAIL) __builtin_amdgcn_sched_barrier(0);
  }
}

template <int DT, int RT, int CT>
__global__ __launch_bounds__(512) void q4_few_kernel(const Q4Args a) {
  extern __shared__ f32x4 part[];  // [waves][2][CT][64]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int r16 = lane & 15, quarter = lane >> 4;
  const uint32_t slot = divide_by(a.by_tiles, blockIdx.x), tile = blockIdx.x - slot * a.by_tiles.d;
  int expert;
  uint32_t first, end;
  if (!find_tile(a, slot, 16 * CT, &expert, &first, &end)) return;
  // Row of weights m0 + 16 rt + r16 of the outputs; with glu, tiles alternate between gate and up rows.
  const int pair = a.glu ? 2 : 1;
  const int64_t m0 = (int64_t)tile * (16 * RT / pair);
  if (expert == a.experts) {
    const uint32_t cols = 16 * RT / pair;
    for (uint32_t i = threadIdx.x; i < 16 * CT * cols; i += blockDim.x) {
      const uint32_t n = first + i / cols;
      const int64_t m = m0 + i % cols;
      if (n < end && m < a.out_rows) store_y<DT>(a, n, m, 0.f);
    }
    return;
  }
  Few<RT, CT> f;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    int64_t m = m0 + 16 * (rt / pair) + r16;
    m = m < a.out_rows ? m : a.out_rows - 1;
    if (pair == 2 && (rt & 1)) m += a.out_rows;
    m += (int64_t)expert * a.M;
    f.codes[rt] = a.codes + m * a.row_bytes + quarter * 16;
    f.groups[rt] = m * a.groups;
  }
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    uint32_t n = first + 16 * ct + r16;
    n = n < end ? n : end - 1;
    int64_t row = a.src ? (int64_t)divide_by(a.by_choices, (uint32_t)a.src[n] & 0x7fffffffu) : (int64_t)n;
    row = row < a.x_rows ? row : a.x_rows - 1;
    f.x[ct] = a.x + row * a.ldx;
  }
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) f.sum[rt][ct] = f32x4{0, 0, 0, 0};
  const int full = a.K / 128, units = (a.K + 128 * kUnit - 1) / (128 * kUnit);
  for (int u = wave; u < units; u += waves) {
    vec16 w[kUnit][RT];
#pragma unroll
    for (int s = 0; s < kUnit; ++s)
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) w[s][rt] = load_codes(a, f.codes[rt], (int64_t)(u * kUnit + s) * 64);
#pragma unroll
    for (int s = 0; s < kUnit; ++s) {
      const int step = u * kUnit + s;
      if (step < full)
        few_step<DT, RT, CT, false>(a, f, w[s], step);
      else if (step * 128 < a.K)
        few_step<DT, RT, CT, true>(a, f, w[s], step);
    }
  }
  // Join the waves' sums, two tiles of weight rows at a time; lane (r16, quarter) has rows 4 quarter .. + 4 of x.
  constexpr int AT = RT < 2 ? RT : 2;
#pragma unroll
  for (int r0 = 0; r0 < RT; r0 += AT) {
    if (r0) __syncthreads();
#pragma unroll
    for (int t = 0; t < AT; ++t)
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) part[((wave * AT + t) * CT + ct) * 64 + lane] = f.sum[r0 + t][ct];
    __syncthreads();
    const int outs = AT / pair * CT * 64;
    for (int i = threadIdx.x; i < outs; i += blockDim.x) {
      const int l = i & 63, ct = (i >> 6) % CT, t = (i >> 6) / CT;
      f32x4 v = {0, 0, 0, 0}, up = {0, 0, 0, 0};
      for (int wv = 0; wv < waves; ++wv) {
        v += part[((wv * AT + t * pair) * CT + ct) * 64 + l];
        if (pair == 2) up += part[((wv * AT + t * pair + 1) * CT + ct) * 64 + l];
      }
      const int64_t m = m0 + 16 * (pair == 2 ? r0 / 2 + t : r0 + t) + (l & 15);
      if (m >= a.out_rows) continue;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t n = first + 16 * ct + 4 * (l >> 4) + k;
        if (n < end) store_y<DT>(a, n, m, pair == 2 ? silu(v[k]) * up[k] : v[k]);
      }
    }
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

template <int RT, int CT>
q4_fn pick_few(int dt) {
  return dt == EBAG_F32 ? q4_few_kernel<0, RT, CT> : dt == EBAG_F16 ? q4_few_kernel<1, RT, CT> : q4_few_kernel<2, RT, CT>;
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
  const bool many = a.rows > 16 * (a.offsets ? h->experts : 1);
  const int rt = 2, ct = many ? 2 : 1;
  const int64_t per_tile = 16 * rt / (h->glu ? 2 : 1);
  const int64_t tiles = (a.out_rows + per_tile - 1) / per_tile;
  const int64_t slots = a.offsets ? most_tiles(a.rows, h->experts, 16 * ct) : (a.rows + 16 * ct - 1) / (16 * ct);
  if (tiles * slots > INT_MAX) return fail(EBAG_EUNSUPPORTED, "too many tiles for one launch");
  a.by_tiles = make_divisor(tiles);
  const int units = (a.K + 128 * kUnit - 1) / (128 * kUnit);
  const int waves = units < 8 ? units : 8;
  const size_t lds = (size_t)waves * 2 * ct * 64 * sizeof(f32x4);
  const q4_fn fn = many ? pick_few<2, 2>(h->dtype) : pick_few<2, 1>(h->dtype);
  hipLaunchKernelGGL(fn, dim3((unsigned)(tiles * slots)), dim3(64 * waves), lds, stream, a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? EBAG_OK : hipf(e, "launch the product with 4-bit weights");
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
  return launch_few(h, a, stream);
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
  return launch_few(h, a, stream);
}

void gemv_ar_q4_destroy(gemv_ar_q4_t h) { delete h; }

}  // extern "C"
