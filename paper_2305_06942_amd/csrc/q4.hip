// Products with 4-bit weights (gemv_ar_q4_* of include/gemv_ar.h): rounding to 4
// bits, and the host side: checks, launch shapes, the choice of kernel.
#include <hip/hip_runtime.h>

#include <climits>
#include <new>

#include "ebag_a2a.h"
#include "gemv_ar.h"
#include "lanes.h"
#include "q4.h"

using namespace ebag;

namespace {

// ------------------------------------------------------------------- to 4 bits

constexpr int kQuantThreads = 256;

struct QuantArgs {
  const char* w;
  uint8_t* codes;
  char* scales;
  uint8_t* zeros;
  int64_t rows;  // of all matrices
  int64_t row_bytes;
  int32_t K, group, groups;
  int32_t lanes;      // that share a group, 2^k <= 64
  Divisor by_groups;
};

// 2^k lanes have a group of a row, 8 columns each at a time: what a lane loads as
// one vector (two in fp32) it stores as one word of codes.  Values of groups of up to
// 512 columns stay in registers between the extremes and the codes.  65536 x 8192
// bf16, groups of 128: 486 us, 2.8 TB/s read and written, bound by the eight exact
// divisions of a lane.
template <int DT>
__global__ __launch_bounds__(kQuantThreads) void q4_quantize_kernel(const QuantArgs a) {
  typedef Type<DT> T;
  typedef typename T::elt elt;
  constexpr int VECS = 8 / T::N;
  const int per_wg = kQuantThreads / a.lanes, own = threadIdx.x / a.lanes, lane = threadIdx.x % a.lanes;
  const int64_t first = (int64_t)blockIdx.x * per_wg, first_row = first / a.groups;
  const uint32_t g_on = (uint32_t)(first - first_row * a.groups) + own, rows_on = divide_by(a.by_groups, g_on);
  const int64_t row = first_row + rows_on;
  if (row >= a.rows) return;  // all lanes of a group together
  const int64_t k0 = (int64_t)(g_on - rows_on * a.groups) * a.group;
  const int64_t k1 = a.K - k0 < a.group ? a.K : k0 + a.group, step = 8 * a.lanes;
  const char* w = a.w + row * a.K * (int64_t)sizeof(elt);
  auto load = [&](float* f, int64_t k) {
    if (k + 8 <= k1) {
#pragma unroll
      for (int i = 0; i < VECS; ++i) T::widen(load16(w + k * (int64_t)sizeof(elt) + 16 * i), f + i * T::N);
      return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = k + i < k1 ? T::widen(reinterpret_cast<const elt*>(w)[k + i]) : 0.f;
  };
  float hi = 0.f, minus_lo = 0.f;
  auto extremes = [&](const float* f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      hi = fmaxf(hi, f[i]);
      minus_lo = fmaxf(minus_lo, -f[i]);
    }
  };
  const int64_t k = k0 + 8 * lane;
  float mine[8], more[8];
  load(mine, k);
  extremes(mine);
  for (int64_t at = k + step; at < k1; at += step) {
    load(more, at);
    extremes(more);
  }
  hi = max_lanes(hi, a.lanes);
  minus_lo = max_lanes(minus_lo, a.lanes);
  const elt scale = T::narrow(a.zeros ? (hi + minus_lo) / 15.f : fmaxf(hi, minus_lo) / 7.f);
  const float s = T::widen(scale);
  float zero = 8.f;
  if (a.zeros) zero = s > 0.f ? fminf(fmaxf(rintf(minus_lo / s), 0.f), 15.f) : 0.f;
  if (lane == 0) {
    const int64_t at = row * a.groups + (g_on - rows_on * a.groups);
    reinterpret_cast<elt*>(a.scales)[at] = scale;
    if (a.zeros) a.zeros[at] = (uint8_t)zero;
  }
  auto store = [&](const float* f, int64_t at) {
    const int have = k1 - at < 8 ? (int)(k1 - at) : 8;
    uint32_t word = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float q = s > 0.f ? rintf(f[i] / s) + zero : zero;
      word |= i < have ? (uint32_t)fminf(fmaxf(q, 0.f), 15.f) << (4 * i) : 0u;
    }
    uint8_t* out = a.codes + row * a.row_bytes + at / 2;  // groups begin at even columns
    if (have == 8)
      __builtin_memcpy(out, &word, 4);
    else
      for (int i = 0; 2 * i < have; ++i) out[i] = (uint8_t)(word >> (8 * i));
  };
  if (k < k1) store(mine, k);
  for (int64_t at = k + step; at < k1; at += step) {
    load(more, at);
    store(more, at);
  }
}

constexpr int kCuLds = 160 * 1024, kCus = 256;

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
  a->by_choices = make_divisor(1);
  a->by_group_blocks = make_divisor(h->group / 32);
  return EBAG_OK;
}

int launch_few(const gemv_ar_q4_plan* h, Q4Args a, bool y32, hipStream_t stream) {
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
  // Its turns: as many workgroups as the card's registers hold at a time, `held` to a CU, so that x is staged once and no
  // place runs empty early (gated, 512 of them: 128 experts of 2 x 1024 x 2048, two rows each, with 512 workgroups 52.1
  // us, 768 55.9, 1024 56.0, 384 61; 64 experts of 4096 x 2048, four rows each, with 512 57.6, 1024 57.8, 2048 60.8, 256
  // 68; the same plain, 1024 of them: with 1024 58.6, 2048 58.8, 512 66.5, 256 94; one fp16 row x 65536 x 8192, 1024 of
  // them: with 1024 56.7, 2048 60.0, 768 65.7).  With experts `slots` is the most tiles that their rows can make: where
  // many have none, fewer workgroups have work (128 gated experts of 2 x 1024 x 2048 with one row each at random, a third
  // of them without: 49.5 us, with 1024 workgroups 44.8).
  const int64_t turn_rows = 16 * (waves / a.split);
  const int64_t all_turns = (a.out_rows + turn_rows - 1) / turn_rows;
  const int64_t held = (rt == 2 ? 8 : parts == 3 ? 12 : 16) / waves;
  int64_t turns = all_turns * slots / (kCus * held);
  turns = turns < 1 ? 1 : turns > all_turns ? all_turns : turns;
  a.turns = (int)turns;
  const int64_t tiles = (all_turns + turns - 1) / turns;
  if (tiles * slots > INT_MAX) return fail(EBAG_EUNSUPPORTED, "too many tiles for one launch");
  a.by_tiles = make_divisor(tiles);
  // LDS for x: all of it up to 40 KiB; or what as many workgroups as a CU gets, or as its registers hold, leave each
  // other; a turn's columns at least (12 x 10000 x 4992 on 625 workgroups: 20.9 us with 49 KB each, 26.8 with 61, 38 with
  // 88; one fp32 row x 4096 x 11008 on 256: all of x at once 14.5 us, 40 KB at a time 19.1; 2 x 65536 x 8192, 33 KB of x:
  // three workgroups on a CU 66 us, four that stage x anew for every tile 78).
  a.all_columns = units * columns;
  const int64_t all_x = (int64_t)rows * parts * (2 * (int64_t)a.all_columns + 16);
  const int64_t least = (int64_t)rows * parts * (2 * a.split * columns + 16);
  const int64_t each = (tiles * slots + kCus - 1) / kCus, on_cu = each < held ? each : held;
  int64_t room = kCuLds / on_cu - (a.split > 1 ? sums : 0) - 16;
  if (room < all_x && all_x <= 40960) room = all_x;
  if (room < least) room = least;
  const int64_t fit = room / (parts * (2 * (int64_t)a.all_columns + 16));
  a.fit_rows = fit < rows ? (int)fit : rows;
  a.some_columns = (int)((room / (rows * parts) - 16) / (2 * a.split * columns)) * a.split * columns;
  a.by_all = make_divisor(a.all_columns / 8);
  a.by_some = make_divisor(a.some_columns / 8);
  const int64_t all = a.fit_rows * parts * (2 * (int64_t)a.all_columns + 16);
  const int64_t some = a.fit_rows < rows ? rows * parts * (2 * (int64_t)a.some_columns + 16) : 0;
  a.x_bytes = (int)(all > some ? all : some);
  const size_t lds = a.x_bytes + (a.split > 1 ? sums : 0);
  const Q4FewKind kind = {rt, whole, a.zeros != nullptr, a.row_bytes % 4 == 0 && reinterpret_cast<uintptr_t>(a.codes) % 4 == 0, y32};
  const q4_fn fn = h->dtype == EBAG_F32 ? pick_q4_few_f32(kind) : h->dtype == EBAG_F16 ? pick_q4_few_f16(kind) : pick_q4_few_bf16(kind);
  hipLaunchKernelGGL(fn, dim3((unsigned)(tiles * slots)), dim3(64 * waves), lds, stream, a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? EBAG_OK : hipf(e, "launch the product with 4-bit weights");
}

int launch_tile(const gemv_ar_q4_plan* h, Q4Args a, bool y32, int x_tiles, hipStream_t stream) {
  const int64_t cols = 32 * x_tiles, per_wg = kQ4TileRows / (h->glu ? 2 : 1);
  const int64_t tiles = (a.out_rows + per_wg - 1) / per_wg;
  const int64_t slots = a.offsets ? most_tiles(a.rows, h->experts, cols) : (a.rows + cols - 1) / cols;
  if (tiles * slots > INT_MAX) return fail(EBAG_EUNSUPPORTED, "too many tiles for one launch");
  a.by_tiles = make_divisor(tiles);
  launch_q4_tile(a, h->dtype, y32, x_tiles, (unsigned)(tiles * slots), stream);
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
// 67.)  fp32 x: 16.5 ns; with 32 rows 235 ns and 64 us, or 272 ns and 85 us (one of 4096 x
// 4096, in us by the two: 64 rows 34, 63; 512 rows 128, 69; 2048 rows 490, 234; with groups
// of 32 523, 279).  bf16 x with an fp32 y takes 1.3 times as long in all three (8192 x 4096, in
// us: 128 rows 49, 65, 85; 256 rows 92, 67, 86; 512 rows 173, 96, 89).  An expert's rows fill their last tile half on average.
int launch(const gemv_ar_q4_plan* h, const Q4Args& a, int y_dtype, hipStream_t stream) {
  const bool y32 = y_dtype == EBAG_F32;
  if (h->K >= 1 << 27) return launch_few(h, a, y32, stream);
  const bool whole = h->group % 128 == 0;
  auto tiles = [&](double rows, double cols) {  // of `rows` weight rows and `cols` rows of x
    const double experts = a.offsets ? h->experts : 1, some = a.rows < experts ? a.rows : experts;
    const double slots = a.offsets ? a.rows / cols + experts / 2 : 0, all = (a.rows + (int)cols - 1) / (int)cols;
    const double n = a.offsets ? (slots < some ? some : slots) : all;
    return (double)((h->M + (int)rows - 1) / (int)rows) * (n < a.rows ? n : a.rows);
  };
  auto at_least = [](double v, double least) { return v < least ? least : v; };
  if (h->dtype == EBAG_F32) {
    const double tile = at_least(tiles(kQ4TileRows, 32) * (whole ? 0.235 : 0.272), whole ? 64 : 85);
    return tiles(16, 16) * 0.0165 <= tile ? launch_few(h, a, y32, stream) : launch_tile(h, a, y32, 1, stream);
  }
  const double few = tiles(16, 16) * (whole ? 0.0080 : 0.0125);
  const double one = at_least(tiles(kQ4TileRows, 32) * 0.157, 45);
  const double two = at_least(tiles(kQ4TileRows, 64) * (whole ? 0.203 : 0.48), whole ? 62 : 107);
  if (few <= two && (few <= one || !whole)) return launch_few(h, a, y32, stream);
  return launch_tile(h, a, y32, whole && one <= two ? 1 : 2, stream);
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
  a.by_groups = make_divisor(a.groups);
  a.lanes = 1;
  while (a.lanes < 64 && 8 * a.lanes < a.group) a.lanes *= 2;
  const int64_t per_wg = kQuantThreads / a.lanes, wgs = (a.rows * a.groups + per_wg - 1) / per_wg;
  if (wgs > INT_MAX) return fail(EBAG_EUNSUPPORTED, "too many groups for one launch");
  void (*fn)(const QuantArgs) = h->dtype == EBAG_F32   ? q4_quantize_kernel<0>
                                : h->dtype == EBAG_F16 ? q4_quantize_kernel<1>
                                                       : q4_quantize_kernel<2>;
  hipLaunchKernelGGL(fn, dim3((unsigned)wgs), dim3(kQuantThreads), 0, stream, a);
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
  return launch(h, a, y_dtype, stream);
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
  return launch(h, a, y_dtype, stream);
}

void gemv_ar_q4_destroy(gemv_ar_q4_t h) { delete h; }

}  // extern "C"
