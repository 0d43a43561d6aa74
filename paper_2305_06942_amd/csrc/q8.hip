// Products in 8-bit integers (gemv_ar_q8_* of include/gemv_ar.h): rounding to 8
// bits, and the host side: checks, launch shapes, the choice of kernel.
#include <hip/hip_runtime.h>

#include <climits>
#include <cmath>
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

// Waves with different rows of weights: as many as leave every CU a workgroup, since they share x; the others share the
// columns (bf16, in us by 1, 2, 4 and 8 of them: 16 rows x 4096 x 4096 6.7, 7.7; x 14336 x 4096 16.8, 13.1; x 65536 x 8192
// 103, 92; 32 rows 8.0, 10.0, 12.7; 20.6, 15.2, 14.7; 135, 104, 95; 64 rows 11.3, 12.7, 17.5, 20.3; 40, 20.3, 19.4, 22.2;
// 238, 136, 109, 97).  One tile of weights to a wave; two, for glu, take 1 to 30 % longer.  Where few workgroups have
// much of K each, eight waves share it.
int launch_few(Q8Args a, int x_tiles, hipStream_t stream) {
  const int cols = 16 * x_tiles;
  const int64_t slots = a.offsets ? most_tiles(a.rows, a.experts, cols) : (a.rows + cols - 1) / cols;
  const int64_t wave_tiles = (a.out_rows + 15) / 16, used = a.offsets ? (a.rows + cols - 1) / cols : slots;
  const int most = x_tiles == 1 ? 2 : x_tiles == 2 ? 4 : 8;
  int waves = x_tiles == 8 ? 4 : 1;
  const int64_t lines = a.pitch / kQ8Line;  // not more waves to the columns than lines (77 rows x 2610 x 94, 17 experts: 44 -> 10 us)
  while (waves < most && (wave_tiles * used >= 200 * 2 * waves || lines * waves < 4)) waves *= 2;
  // A few tiles are not an eighth for each XCD: they are left to all of them (2920 rows x 54 x 2587: 15.3 -> 7.7 us).
  const int64_t grid_tiles = (wave_tiles + waves - 1) / waves;
  a.spread = grid_tiles < 64 ? 0 : 3;
  const int64_t eighths = ((grid_tiles - 1) >> a.spread) + 1;
  const int64_t group = !a.spread ? 1 : a.offsets ? (a.rows > (int64_t)cols * a.experts ? 4 : 1) : slots < 8 ? slots : 8, groups = (slots + group - 1) / group;
  const int64_t grid = (eighths << a.spread) * group * groups;
  if (grid > UINT32_MAX / 512) return fail(EBAG_EUNSUPPORTED, "too many tiles for one launch");
  a.by_tiles = make_divisor(eighths);
  a.tiles = (uint32_t)grid_tiles;
  a.by_group = make_divisor(group);
  if (a.x)
    launch_q8_own(a, a.glu ? 2 : 1, waves, (unsigned)grid, stream);
  else
    launch_q8_few(a, a.glu ? 2 : 1, x_tiles, waves, (unsigned)grid, stream);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? EBAG_OK : hipf(e, "launch the product in 8 bits");
}

int launch_tile(Q8Args a, Q8Tile kind, hipStream_t stream) {
  const int x_rows = q8_tile_x(kind);
  const int64_t per_wg = q8_tile_w(kind) / (a.glu ? 2 : 1), tiles = (a.out_rows + per_wg - 1) / per_wg;
  const int64_t slots = a.offsets ? most_tiles(a.rows, a.experts, x_rows) : (a.rows + x_rows - 1) / x_rows;
  const int64_t grid = (slots + 3) / 4 * 4 * tiles;
  if (grid > UINT32_MAX / 512) return fail(EBAG_EUNSUPPORTED, "too many tiles for one launch");
  a.by_tiles = make_divisor(tiles);
  a.whole = (uint32_t)(grid / 256 * 256);
  launch_q8_tile(a, kind, (unsigned)grid, stream);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? EBAG_OK : hipf(e, "launch the product in 8 bits");
}

// Which kernel, by a model of measured times in us.  A kernel has `cols` rows of x and `rows` of weights to a workgroup.
// `fix` is its beginning and end; K = 4096 (times K / 4096 for others) takes at least `least`, a workgroup's own time, and
// otherwise `start` and `each` ns for every 16 x 16 sums, or `round` for every 256 workgroups of the largest tiles, one
// to a CU.  With a shorter K the results' own time shows, `ends` ns for 16 x 16 of them, and the largest tiles take at
// least `floor`.  Where the weights are more than the caches hold, memory's rate bounds all of them, `rate` in TB/s, at 1.5 times
// the bytes with two tiles of x and so on in the kernel that streams (its tiles of x share weights in the L2 by half).
// Fitted to 129 products in bf16 with every kernel, K from 80 to 10128: what it takes is 1 % slower than the fastest of the
// seven on average, 33 % at most.  Some of them, in us by 16, 32, 64 and 128 rows of x in the streaming kernel, 256 x 64,
// 512 x 128 and 256 x 256:
//   4096 x 4096: 64 rows 9.5, 9.9, 11.5, 24, 20.3, 48, 45; 256 rows 25, 16.7, 18.3, 27, 21, 50, 48; 512 rows 45, 30.5, 20, 28.5, 22.7,
//     50, 48; 2048 rows 167, 88, 56, 63, 41, 56, 52
//   128 rows x 65536 x 8192: 354, 206, 143, 120, 194, 215, 347; 512 rows x 20000 x 256: 56, 27, 21, 30, 14, 18, 27
//   2920 rows x 54 x 2587: 7.7, 10.4, 11.8, 20, 17, 44, 42
//   gated experts of 2 x 1024 x 2048: 128 of them with 2 rows each 85, 88, 214, 140, 85, 98, 133; 64 with 32 rows each 88, 62,
//     65, 88, 53, 58, 74; of 2 x 2048 x 2048, 64 with 512 rows each 1724, 850, 648, 568, 387, 377, 384
struct Kernel {
  int x_tiles;  // of 16 rows, in the streaming kernel; 0: the matrix-product kernel
  Q8Tile tile;
  double cols, rows, fix, floor, least, start, each, ends, round, rate;
};
constexpr Kernel kKernels[] = {
    {1, Q8_256x64, 16, 16, 3.1, 0, 3.6, 1, 4.4, 1.7, 0, 5.6},      {2, Q8_256x64, 32, 16, 3.9, 0, 3.3, 4.1, 2.1, 0.5, 0, 5.6},
    {4, Q8_256x64, 64, 16, 5.2, 0, 4.8, 4.3, 1.9, 0.3, 0, 5.6},    {8, Q8_256x64, 128, 16, 4.9, 0, 22, 0, 1.6, 0.45, 0, 4.5},
    {0, Q8_256x64, 64, 256, 5.3, 0, 18, 2.5, 0.9, 0.18, 0, 5.4},   {0, Q8_512x128, 128, 512, 4.2, 17, 42, 0, 0, 0.3, 58, 2.5},
    {0, Q8_256x256, 256, 256, 7.5, 14, 43, 0, 0, 0.25, 50, 1.5}};

double time_of(const Kernel& k, const Q8Args& a) {
  const double M = (double)a.M, scale = (double)a.pitch / 4096;
  const double used = a.offsets ? (a.rows < (uint32_t)a.experts ? a.rows : a.experts) : 1;  // matrices with rows
  const double per = (double)a.rows / used;
  // Tiles of x: an expert's last one is half full on average.
  double slots = a.offsets ? a.rows / k.cols + used / 2 : std::ceil(a.rows / k.cols);
  slots = slots < used ? used : slots;
  const double wgs = std::ceil(M / k.rows) * slots, sums = std::ceil(M / k.rows) * (k.rows / 16) * slots * (k.cols / 16);
  double t = k.round ? std::ceil(wgs / 256) * k.round : k.start + sums * k.each * 1e-3;
  t = k.fix + scale * (t < k.least ? k.least : t);
  if (scale < 1) t += sums * k.ends * 1e-3 * (1 - scale);
  if (t < k.floor) t = k.floor;
  const double bytes = used * M * (double)a.pitch;
  if (bytes > 128e6) {
    double memory = bytes / (k.rate * 1e6);
    if (k.x_tiles) memory *= (1 + 0.5 * (std::ceil(per / k.cols) - 1)) * (a.offsets && k.x_tiles > 1 ? 1.25 : 1);
    // One workgroup on a CU, or two that share weights, have too few loads under way.
    if (!k.x_tiles && !k.round && (wgs < 512 || (!a.offsets && per > k.cols))) memory *= 2;
    if (memory > t) t = memory;
  }
  return t;
}

int launch(const Q8Args& a, hipStream_t stream) {
  if (a.x) return launch_few(a, 1, stream);
  const Kernel* best = nullptr;
  double least = 0;
  for (const Kernel& k : kKernels) {
    const double t = time_of(k, a);
    if (!best || t < least) best = &k, least = t;
  }
  return best->x_tiles ? launch_few(a, best->x_tiles, stream) : launch_tile(a, best->tile, stream);
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
  if (!q8_own_fits(a)) {
    if (x)
      if (int rc = launch_round(h, x, ldx, rows, xq, xs, stream)) return rc;
    a.x = nullptr;
  }
  return launch(a, stream);
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
  a.x = nullptr;
  if (x)
    if (int rc = launch_round(h, x, ldx, x_rows, xq, xs, stream)) return rc;
  return launch(a, stream);
}

void gemv_ar_q8_destroy(gemv_ar_q8_t h) { delete h; }

}  // extern "C"
