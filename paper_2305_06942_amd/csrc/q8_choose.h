// Which kernel a product in 8-bit integers takes, and its launch.  Host code, for any compiler.
#pragma once

#include <stdint.h>

#include <cmath>

#include "tiles.h"

namespace ebag {

// Bytes of a row of codes: whole cache lines, so that rows begin on one and every
// step of a product is whole.  Rows of x end in zeros, so what stands behind a
// row of weights does not matter.
constexpr int64_t kQ8Line = 128;
constexpr int64_t q8_pitch(int64_t K) { return (K + kQ8Line - 1) / kQ8Line * kQ8Line; }

// What the choice goes by.
struct Q8Call {
  int64_t M, out_rows, pitch;  // as in Q8Args
  uint32_t rows;
  int32_t experts;
  bool sorted;                 // rows by expert
  bool glu;
};

// Rows of weights and rows of x of a workgroup of the matrix-product kernel.
enum Q8Tile { Q8_256x64, Q8_512x128, Q8_256x256 };
constexpr int q8_tile_w(Q8Tile t) { return t == Q8_512x128 ? 512 : 256; }
constexpr int q8_tile_x(Q8Tile t) { return t == Q8_256x64 ? 64 : t == Q8_512x128 ? 128 : 256; }

constexpr int kQ8OwnWaves = 8;  // of a workgroup that rounds its row of x itself; half of them with glu
constexpr int q8_few_threads(int x_tiles, int waves) { return x_tiles >= 4 && waves == 8 ? 512 : 256; }

struct Q8Shape {
  int64_t grid;
  int threads;
  int64_t tiles;  // workgroups that share the rows of x: of the kernel for few rows those of an XCD, or all
  // The kernel for few rows.
  int waves, spread;
  int64_t all_tiles, group;
  // Threads of a launch are numbered in 32 bits.
  bool fits() const { return grid <= UINT32_MAX / threads; }
};

// Waves with different rows of weights: as many as leave every CU a workgroup, since they share x; the others share the
// columns (bf16, in us by 1, 2, 4 and 8 of them: 16 rows x 4096 x 4096 6.7, 7.7; x 14336 x 4096 16.8, 13.1; x 65536 x 8192
// 103, 92; 32 rows 8.0, 10.0, 12.7; 20.6, 15.2, 14.7; 135, 104, 95; 64 rows 11.3, 12.7, 17.5, 20.3; 40, 20.3, 19.4, 22.2;
// 238, 136, 109, 97).  One tile of weights to a wave; two, for glu, take 1 to 30 % longer.  Where few workgroups have
// much of K each, eight waves share it.
inline Q8Shape q8_few_shape(const Q8Call& a, int x_tiles, bool own) {
  Q8Shape s{};
  const int cols = 16 * x_tiles;
  const int64_t slots = a.sorted ? most_tiles(a.rows, a.experts, cols) : ((int64_t)a.rows + cols - 1) / cols;
  const int64_t wave_tiles = (a.out_rows + 15) / 16, used = a.sorted ? ((int64_t)a.rows + cols - 1) / cols : slots;
  const int most = x_tiles == 1 ? 2 : x_tiles == 2 ? 4 : 8;
  s.waves = x_tiles == 8 ? 4 : 1;
  const int64_t lines = a.pitch / kQ8Line;  // not more waves to the columns than lines (77 rows x 2610 x 94, 17 experts: 44 -> 10 us)
  while (s.waves < most && (wave_tiles * used >= 200 * 2 * s.waves || lines * s.waves < 4)) s.waves *= 2;
  s.threads = own ? 64 * kQ8OwnWaves / (a.glu ? 2 : 1) : q8_few_threads(x_tiles, s.waves);
  // A few tiles are not an eighth for each XCD: they are left to all of them (2920 rows x 54 x 2587: 15.3 -> 7.7 us).
  s.all_tiles = (wave_tiles + s.waves - 1) / s.waves;
  s.spread = s.all_tiles < 64 ? 0 : 3;
  s.tiles = ((s.all_tiles - 1) >> s.spread) + 1;
  // Slots that have their turn with a workgroup's weights, which are then in the L2 (16 rows of x to a slot, in us by 1, 2, 4 and 8
  // slots: 64 rows x 65536 x 8192 356, 257, 206, 206; 128 rows 710, 504, 405, 357; x 20000 x 4096 64 rows 49, 31, 28, 28).  Rows by expert
  // have few slots to a matrix, and nothing to gain or lose (4096 rows on 128 experts of 1024 x 2048 83.5, 83.2, 80.8, 86.2).
  s.group = !s.spread ? 1 : a.sorted ? (a.rows > (int64_t)cols * a.experts ? 4 : 1) : slots < 8 ? slots : 8;
  s.grid = (s.tiles << s.spread) * s.group * ((slots + s.group - 1) / s.group);
  return s;
}

inline Q8Shape q8_tile_shape(const Q8Call& a, Q8Tile kind) {
  Q8Shape s{};
  const int x_rows = q8_tile_x(kind);
  const int64_t per_wg = q8_tile_w(kind) / (a.glu ? 2 : 1);
  const int64_t slots = a.sorted ? most_tiles(a.rows, a.experts, x_rows) : ((int64_t)a.rows + x_rows - 1) / x_rows;
  s.tiles = (a.out_rows + per_wg - 1) / per_wg;
  s.grid = (slots + 3) / 4 * 4 * s.tiles;
  s.threads = 256;
  return s;
}

// Which kernel, by a model of measured times in us.  A kernel has `cols` rows of x and `rows` of weights to a workgroup.
// `fix` is its beginning and end; K = 4096 (times K / 4096 for others) takes at least `least`, a workgroup's own time, and
// otherwise `start` and `each` ns for every 16 x 16 sums, or `round` for every 256 workgroups of the largest tiles, one
// to a CU.  With a shorter K the results' own time shows, `ends` ns for 16 x 16 of them, and the largest tiles take at
// least `floor`.  Where the weights are more than the caches hold, memory's rate bounds all of them, `rate` in TB/s, at 1.5 times
// the bytes with two tiles of x and so on in the kernel that streams (its tiles of x share weights in the L2 by half).
// Fitted to 129 products in bf16 with every kernel, K from 80 to 10128: of these, what it takes is 1 % slower than the fastest
// of the seven on average, 33 % at most.  An fp32 y and experts of uneven popularity are not among them; how the rows
// lie over the experts it does not know.  Some of them, in us by 16, 32, 64 and 128 rows of x in the streaming kernel, 256 x 64,
// 512 x 128 and 256 x 256:
//   4096 x 4096: 64 rows 9.5, 9.9, 11.5, 24, 20.3, 48, 45; 256 rows 25, 16.7, 18.3, 27, 21, 50, 48; 512 rows 45, 30.5, 20, 28.5, 22.7,
//     50, 48; 2048 rows 167, 88, 56, 63, 41, 56, 52
//   128 rows x 65536 x 8192: 354, 206, 143, 120, 194, 215, 347; 512 rows x 20000 x 256: 56, 27, 21, 30, 14, 18, 27
//   2920 rows x 54 x 2587: 7.7, 10.4, 11.8, 20, 17, 44, 42
//   gated experts of 2 x 1024 x 2048: 128 of them with 2 rows each 85, 88, 214, 140, 85, 98, 133; 64 with 32 rows each 88, 62,
//     65, 88, 53, 58, 74; of 2 x 2048 x 2048, 64 with 512 rows each 1724, 850, 648, 568, 387, 377, 384
struct Q8Kernel {
  int x_tiles;  // of 16 rows, in the streaming kernel; 0: the matrix-product kernel
  Q8Tile tile;
  double cols, rows, fix, floor, least, start, each, ends, round, rate;
};
constexpr Q8Kernel kQ8Kernels[] = {
    {1, Q8_256x64, 16, 16, 3.1, 0, 3.6, 1, 4.4, 1.7, 0, 5.6},      {2, Q8_256x64, 32, 16, 3.9, 0, 3.3, 4.1, 2.1, 0.5, 0, 5.6},
    {4, Q8_256x64, 64, 16, 5.2, 0, 4.8, 4.3, 1.9, 0.3, 0, 5.6},    {8, Q8_256x64, 128, 16, 4.9, 0, 22, 0, 1.6, 0.45, 0, 4.5},
    {0, Q8_256x64, 64, 256, 5.3, 0, 18, 2.5, 0.9, 0.18, 0, 5.4},   {0, Q8_512x128, 128, 512, 4.2, 17, 42, 0, 0, 0.3, 58, 2.5},
    {0, Q8_256x256, 256, 256, 7.5, 14, 43, 0, 0, 0.25, 50, 1.5}};

inline double q8_time(const Q8Kernel& k, const Q8Call& a) {
  const double M = (double)a.M, scale = (double)a.pitch / 4096;
  const double used = a.sorted ? (a.rows < (uint32_t)a.experts ? a.rows : a.experts) : 1;  // matrices with rows
  const double per = (double)a.rows / used;
  // Tiles of x: an expert's last one is half full on average.
  double slots = a.sorted ? a.rows / k.cols + used / 2 : std::ceil(a.rows / k.cols);
  slots = slots < used ? used : slots;
  const double wgs = std::ceil(M / k.rows) * slots, sums = std::ceil(M / k.rows) * (k.rows / 16) * slots * (k.cols / 16);
  double t = k.round ? std::ceil(wgs / 256) * k.round : k.start + sums * k.each * 1e-3;
  t = k.fix + scale * (t < k.least ? k.least : t);
  if (scale < 1) t += sums * k.ends * 1e-3 * (1 - scale);
  if (t < k.floor) t = k.floor;
  const double bytes = used * M * (double)a.pitch;
  if (bytes > 128e6) {
    double memory = bytes / (k.rate * 1e6);
    if (k.x_tiles) memory *= (1 + 0.5 * (std::ceil(per / k.cols) - 1)) * (a.sorted && k.x_tiles > 1 ? 1.25 : 1);
    // One workgroup on a CU, or two that share weights, have too few loads under way.
    if (!k.x_tiles && !k.round && (wgs < 512 || (!a.sorted && per > k.cols))) memory *= 2;
    if (memory > t) t = memory;
  }
  return t;
}

inline Q8Shape q8_shape(const Q8Call& a, const Q8Kernel& k) {
  return k.x_tiles ? q8_few_shape(a, k.x_tiles, false) : q8_tile_shape(a, k.tile);
}

// The fastest of those whose launch holds the product; nullptr: there is none, which takes M above 2^30 or more memory
// than the card has.
inline const Q8Kernel* q8_choose(const Q8Call& a) {
  constexpr int kKernels = sizeof kQ8Kernels / sizeof *kQ8Kernels;
  bool out[kKernels] = {};
  for (;;) {
    int best = -1;
    double least = 0;
    for (int i = 0; i < kKernels; ++i) {
      if (out[i]) continue;
      const double t = q8_time(kQ8Kernels[i], a);
      if (best < 0 || t < least) best = i, least = t;
    }
    if (best < 0) return nullptr;
    if (q8_shape(a, kQ8Kernels[best]).fits()) return &kQ8Kernels[best];
    out[best] = true;
  }
}

}  // namespace ebag
