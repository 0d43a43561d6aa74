// Products in 8-bit integers (gemv_ar_q8_* of include/gemv_ar.h): rounding to 8
// bits, and the host side: checks, launch shapes, the choice of kernel.
#include <hip/hip_runtime.h>

#include <climits>
#include <new>

#include "ebag_a2a.h"
#include "gemv_ar.h"
#include "q8.h"

using namespace ebag;

namespace {

// ------------------------------------------------------------------- to 8 bits

constexpr int kRoundThreads = 256;
constexpr int kHeld = 4;  // units of 8 elements that a lane holds

struct RoundArgs {
  const char* x;
  int8_t* codes;
  float* scales;
  int64_t ld;       // bytes
  int64_t pitch;
  int64_t rows;
  int32_t K;
  int32_t units;    // of 8 elements, the last one short or empty: pitch / 8
};

// WAVE: a wave to a row, otherwise a workgroup.  Up to 32 elements of a lane stay in registers between
// the largest and the codes; longer rows are read again.  Bound by memory: 8192 rows of 8192 bf16, 201 MB, 45 us or 4.5 TB/s.
template <int DT, bool WAVE>
__global__ __launch_bounds__(WAVE ? kRoundThreads : 1024) void q8_round_kernel(const RoundArgs a) {
  __shared__ uint32_t tops[16];
  const int lanes = WAVE ? 64 : blockDim.x, lane = WAVE ? threadIdx.x % 64 : threadIdx.x;
  const int64_t row = WAVE ? (int64_t)blockIdx.x * (kRoundThreads / 64) + threadIdx.x / 64 : blockIdx.x;
  if (WAVE && row >= a.rows) return;
  const char* x = a.x + row * a.ld;
  int8_t* codes = a.codes + row * a.pitch;
  float held[kHeld][8];
  uint32_t top = 0;
  auto look = [&](const float* f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t v = __float_as_uint(f[i]) & 0x7fffffffu;
      top = top > v ? top : v;
    }
  };
#pragma unroll
  for (int u = 0; u < kHeld; ++u) {
    const int unit = u * lanes + lane;
    if (unit < a.units) {
      q8_load8<DT>(x, unit * 8, a.K, held[u]);
      look(held[u]);
    }
  }
  for (int unit = kHeld * lanes + lane; unit < a.units; unit += lanes) {
    float f[8];
    q8_load8<DT>(x, unit * 8, a.K, f);
    look(f);
  }
  top = q8_largest(top);
  if (!WAVE) {
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 16; ++w)
      if (w < (int)blockDim.x / 64) top = top > tops[w] ? top : tops[w];
  }
  const float scale = q8_scale(top);
  if (lane == 0) a.scales[row] = scale;
  const Q8Rounder r(scale);
#pragma unroll
  for (int u = 0; u < kHeld; ++u) {
    const int unit = u * lanes + lane;
    if (unit < a.units) q8_store8(codes + unit * 8, r, held[u]);
  }
  for (int unit = kHeld * lanes + lane; unit < a.units; unit += lanes) {
    float f[8];
    q8_load8<DT>(x, unit * 8, a.K, f);
    q8_store8(codes + unit * 8, r, f);
  }
}

int hipf(hipError_t e, const char* what) { return fail(EBAG_EHIP, "%s: %s", what, hipGetErrorString(e)); }

}  // namespace

struct gemv_ar_q8_plan {
  int device = 0;
  int64_t M = 0, K = 0, pitch = 0;
  int32_t dtype = 0, experts = 0, glu = 0;
};

namespace {

int check_plan(const gemv_ar_q8_plan* h) {
  if (!h) return fail(EBAG_EINVAL, "null plan");
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev != h->device)
    return fail(EBAG_EINVAL, "the plan belongs to device %d, but device %d is current", h->device, dev);
  return EBAG_OK;
}

int elt_of(int dtype) { return dtype == EBAG_F32 ? 4 : 2; }

int check_x(const gemv_ar_q8_plan* h, const void* x, int64_t ldx, const int8_t* xq, const float* xs) {
  if (!xq || !xs) return fail(EBAG_EINVAL, "null xq or xs");
  if (reinterpret_cast<uintptr_t>(xq) % 16 || reinterpret_cast<uintptr_t>(xs) % 4)
    return fail(EBAG_EINVAL, "xq not aligned to 16 bytes or xs not to its elements");
  if (!x) return EBAG_OK;
  if (reinterpret_cast<uintptr_t>(x) % elt_of(h->dtype)) return fail(EBAG_EINVAL, "x not aligned to its elements");
  if (ldx < h->K || ldx > (int64_t)1 << 40) return fail(EBAG_EINVAL, "row step %lld of x below K=%lld", (long long)ldx, (long long)h->K);
  return EBAG_OK;
}

int launch_round(const gemv_ar_q8_plan* h, const void* x, int64_t ldx, int64_t rows, int8_t* xq, float* xs, hipStream_t stream) {
  RoundArgs a{};
  a.x = static_cast<const char*>(x);
  a.codes = xq;
  a.scales = xs;
  a.ld = ldx * elt_of(h->dtype);
  a.pitch = h->pitch;
  a.rows = rows;
  a.K = (int32_t)h->K;
  a.units = (int32_t)(h->pitch / 8);
  // A wave to a row where rows are short or many (bf16, in us by a wave and by a workgroup: 64 rows of 256 3.2, 3.3, of 1024 4.3,
  // 3.4, of 2048 6.0, 3.5; 1024 rows of 512 3.3, 3.7, of 1024 4.2, 3.9, of 2048 6.1, 4.4; 2048 rows of 512 3.4, 4.5, of 1024 4.5, 5.0, of 2048
  // 6.5, 5.9; 4096 rows of 2048 8.4, 9.1; 16384 rows of 128 7.1, 16.1, of 2048 23.0, 25.7).
  const bool wave = h->K <= 64 * 8 * kHeld && (rows >= 2048 || h->K <= 256);
  const int64_t per_wg = wave ? kRoundThreads / 64 : 1;
  void (*fn)(const RoundArgs) = h->dtype == EBAG_F32   ? wave ? q8_round_kernel<0, true> : q8_round_kernel<0, false>
                                : h->dtype == EBAG_F16 ? wave ? q8_round_kernel<1, true> : q8_round_kernel<1, false>
                                : wave                 ? q8_round_kernel<2, true>
                                                       : q8_round_kernel<2, false>;
  // A few long rows: a thread for every 8 elements, up to 1024 (64 rows of 8192 bf16 with 256 threads each 6.7 us).
  int threads = kRoundThreads;
  while (!wave && rows < 1024 && threads < 1024 && threads < a.units) threads *= 2;
  constexpr int64_t kMost = 1 << 22;  // workgroups of a launch, whose threads are numbered in 32 bits
  for (int64_t left = rows; left > 0; left -= kMost * per_wg) {
    const int64_t wgs = (left + per_wg - 1) / per_wg;
    hipLaunchKernelGGL(fn, dim3((unsigned)(wgs < kMost ? wgs : kMost)), dim3(threads), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return hipf(e, "launch the rounding to 8 bits");
    a.x += kMost * per_wg * a.ld;
    a.codes += kMost * per_wg * a.pitch;
    a.scales += kMost * per_wg;
    a.rows -= kMost * per_wg;
  }
  return EBAG_OK;
}

int fill_args(const gemv_ar_q8_plan* h, const int8_t* codes, const float* scales, const void* x, int64_t ldx, int64_t x_rows,
              const int8_t* xq, const float* xs, int64_t rows, void* y, int64_t ldy, int32_t y_dtype, Q8Args* a) {
  if (y_dtype != h->dtype && y_dtype != EBAG_F32)
    return fail(EBAG_EINVAL, "y_dtype must be fp32 or the plan's type, not %d", (int)y_dtype);
  if (!codes || !scales || !y) return fail(EBAG_EINVAL, "null codes, scales or y");
  if (int rc = check_x(h, x, ldx, xq, xs)) return rc;
  const int y_elt = elt_of(y_dtype);
  const int64_t wide = h->glu ? h->M / 2 : h->M;
  if (reinterpret_cast<uintptr_t>(codes) % 16) return fail(EBAG_EINVAL, "codes not aligned to 16 bytes");
  if (reinterpret_cast<uintptr_t>(scales) % 4 || reinterpret_cast<uintptr_t>(y) % y_elt)
    return fail(EBAG_EINVAL, "scales or y not aligned to its elements");
  if (ldy < wide || ldy > (int64_t)1 << 40) return fail(EBAG_EINVAL, "row step %lld of y below its %lld columns", (long long)ldy, (long long)wide);
  *a = Q8Args{};
  a->codes = codes;
  a->scales = scales;
  a->x = static_cast<const char*>(x);
  a->x_type = h->dtype;
  a->K = (int32_t)h->K;
  a->xq = xq;
  a->xs = xs;
  a->y = static_cast<char*>(y);
  a->ldy = ldy * y_elt;
  a->pitch = h->pitch;
  a->M = h->M;
  a->out_rows = wide;
  a->x_rows = x_rows;
  a->rows = (uint32_t)rows;
  a->experts = h->experts;
  a->glu = h->glu;
  a->y_type = y_dtype;
  a->by_choices = make_divisor(1);
  return EBAG_OK;
}

Q8Call call_of(const Q8Args& a) {
  return Q8Call{a.M, a.out_rows, a.pitch, a.rows, a.experts, a.offsets != nullptr, a.glu != 0};
}

void launch_few(Q8Args a, const Q8Shape& s, int x_tiles, hipStream_t stream) {
  a.by_tiles = make_divisor(s.tiles);
  a.spread = s.spread;
  a.tiles = (uint32_t)s.all_tiles;
  a.by_group = make_divisor(s.group);
  if (a.x)
    launch_q8_own(a, a.glu ? 2 : 1, s.waves, (unsigned)s.grid, stream);
  else
    launch_q8_few(a, a.glu ? 2 : 1, x_tiles, s.waves, (unsigned)s.grid, stream);
}

void launch_tile(Q8Args a, const Q8Shape& s, Q8Tile kind, hipStream_t stream) {
  a.by_tiles = make_divisor(s.tiles);
  a.whole = (uint32_t)(s.grid / 256 * 256);
  launch_q8_tile(a, kind, (unsigned)s.grid, stream);
}

// The product, its rows rounded first where x is given and the product does not do that itself.  The kernel is chosen
// before anything is launched.
int multiply(const gemv_ar_q8_plan* h, Q8Args a, int64_t ldx, int8_t* xq, float* xs, hipStream_t stream) {
  const Q8Call call = call_of(a);
  if (q8_own_fits(a)) {
    launch_few(a, q8_few_shape(call, 1, true), 1, stream);
  } else {
    const Q8Kernel* k = q8_choose(call);
    if (!k) return fail(EBAG_EUNSUPPORTED, "too many tiles for one launch: M=%lld, rows=%u", (long long)a.M, a.rows);
    if (a.x)
      if (int rc = launch_round(h, a.x, ldx, a.x_rows, xq, xs, stream)) return rc;
    a.x = nullptr;
    const Q8Shape s = q8_shape(call, *k);
    k->x_tiles ? launch_few(a, s, k->x_tiles, stream) : launch_tile(a, s, k->tile, stream);
  }
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? EBAG_OK : hipf(e, "launch the product in 8 bits");
}

}  // namespace

extern "C" {

int gemv_ar_q8_create(gemv_ar_q8_t* out, int64_t M, int64_t K, int32_t dtype, int32_t experts, int32_t glu) {
  if (!out) return fail(EBAG_EINVAL, "null output handle");
  *out = nullptr;
  if (M < 1 || M > INT_MAX) return fail(EBAG_EINVAL, "M=%lld outside [1, 2^31)", (long long)M);
  if (K < 1 || K > 1 << 17) return fail(EBAG_EINVAL, "K=%lld outside [1, 2^17]", (long long)K);
  if (dtype != EBAG_F32 && dtype != EBAG_F16 && dtype != EBAG_BF16) return fail(EBAG_EINVAL, "bad dtype %d", (int)dtype);
  if (experts < 1 || experts > 512) return fail(EBAG_EINVAL, "experts=%d outside [1, 512]", experts);
  if (glu != 0 && glu != 1) return fail(EBAG_EINVAL, "glu must be 0 or 1");
  if (glu && M % 2) return fail(EBAG_EINVAL, "glu needs an even M, not %lld", (long long)M);
  gemv_ar_q8_plan* h = new (std::nothrow) gemv_ar_q8_plan();
  if (!h) return fail(EBAG_ENOMEM, "host allocation failed");
  const hipError_t e = hipGetDevice(&h->device);
  if (e != hipSuccess) {
    delete h;
    return hipf(e, "query device");
  }
  h->M = M;
  h->K = K;
  h->pitch = q8_pitch(K);
  h->dtype = dtype;
  h->experts = experts;
  h->glu = glu;
  *out = h;
  clear_error();
  return EBAG_OK;
}

int64_t gemv_ar_q8_pitch(gemv_ar_q8_t h) { return h ? h->pitch : 0; }

int gemv_ar_q8_quantize(gemv_ar_q8_t h, const void* w, int8_t* codes, float* scales, hipStream_t stream) {
  if (int rc = check_plan(h)) return rc;
  if (!w || !codes || !scales) return fail(EBAG_EINVAL, "null w, codes or scales");
  if (reinterpret_cast<uintptr_t>(codes) % 16) return fail(EBAG_EINVAL, "codes not aligned to 16 bytes");
  if (reinterpret_cast<uintptr_t>(w) % elt_of(h->dtype) || reinterpret_cast<uintptr_t>(scales) % 4)
    return fail(EBAG_EINVAL, "w or scales not aligned to its elements");
  return launch_round(h, w, h->K, h->M * h->experts, codes, scales, stream);
}

int gemv_ar_q8_round(gemv_ar_q8_t h, const void* x, int64_t ldx, int64_t rows, int8_t* xq, float* xs, hipStream_t stream) {
  if (int rc = check_plan(h)) return rc;
  if (rows < 0 || rows > INT_MAX) return fail(EBAG_EINVAL, "rows=%lld outside [0, 2^31)", (long long)rows);
  if (!rows) return EBAG_OK;
  if (!x) return fail(EBAG_EINVAL, "null x");
  if (int rc = check_x(h, x, ldx, xq, xs)) return rc;
  return launch_round(h, x, ldx, rows, xq, xs, stream);
}

int gemv_ar_q8_forward(gemv_ar_q8_t h, const int8_t* codes, const float* scales, const void* x, int64_t ldx, int64_t rows,
                       int8_t* xq, float* xs, void* y, int64_t ldy, int32_t y_dtype, hipStream_t stream) {
  if (int rc = check_plan(h)) return rc;
  if (rows < 0 || rows > INT_MAX) return fail(EBAG_EINVAL, "rows=%lld outside [0, 2^31)", (long long)rows);
  if (!rows) return EBAG_OK;
  Q8Args a;
  if (int rc = fill_args(h, codes, scales, x, ldx, rows, xq, xs, rows, y, ldy, y_dtype, &a)) return rc;
  return multiply(h, a, ldx, xq, xs, stream);
}

int gemv_ar_q8_experts(gemv_ar_q8_t h, const int8_t* codes, const float* scales, const void* x, int64_t ldx, int64_t x_rows,
                       int8_t* xq, float* xs, const int32_t* offsets, const int32_t* src, int32_t choices, int64_t rows,
                       void* y, int64_t ldy, int32_t y_dtype, hipStream_t stream) {
  if (int rc = check_plan(h)) return rc;
  if (rows < 0 || rows > INT_MAX) return fail(EBAG_EINVAL, "rows=%lld outside [0, 2^31)", (long long)rows);
  if (!rows) return EBAG_OK;
  if (!offsets) return fail(EBAG_EINVAL, "null offsets");
  if (src && choices < 1) return fail(EBAG_EINVAL, "choices=%d must be positive", choices);
  if (x_rows < 1 || x_rows > INT_MAX || (!src && x_rows != rows))
    return fail(EBAG_EINVAL, "x_rows=%lld: without src x has as many rows as y", (long long)x_rows);
  Q8Args a;
  if (int rc = fill_args(h, codes, scales, x, ldx, x_rows, xq, xs, rows, y, ldy, y_dtype, &a)) return rc;
  a.offsets = offsets;
  a.src = src;
  a.by_choices = make_divisor(src ? choices : 1);
  return multiply(h, a, ldx, xq, xs, stream);
}

void gemv_ar_q8_destroy(gemv_ar_q8_t h) { delete h; }

}  // extern "C"
