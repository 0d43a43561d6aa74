// Host check of the choice of kernel for products in 8-bit integers: a launch's
// threads are numbered in 32 bits, its workgroups cover every tile, no other
// kernel whose launch holds the product is faster by the model, and whatever fits
// the card's memory has a kernel, with M up to 2^30.
#include <cstdint>
#include <cstdio>
#include <random>

#include "q8_choose.h"

using namespace ebag;

int bad = 0, cases = 0;

void say(const Q8Call& a, const char* what) {
  if (++bad < 20)
    std::printf("%s: M=%lld out=%lld pitch=%lld rows=%u experts=%d sorted=%d glu=%d\n", what, (long long)a.M, (long long)a.out_rows,
                (long long)a.pitch, a.rows, a.experts, (int)a.sorted, (int)a.glu);
}

void check(int64_t M, int64_t K, int64_t rows, int32_t experts, bool sorted, bool glu) {
  if (glu && M % 2) ++M;
  const Q8Call a{M, glu ? M / 2 : M, q8_pitch(K), (uint32_t)rows, experts, sorted, glu};
  ++cases;
  const Q8Kernel* k = q8_choose(a);
  const double bytes = (double)experts * M * (a.pitch + 4) + (double)rows * (a.pitch + 4 + 2.0 * a.out_rows);
  if (!k) {
    if (bytes <= 288e9 * 1.08 && M <= 1 << 30) say(a, "no kernel");
    return;
  }
  const Q8Shape s = q8_shape(a, *k);
  if (s.grid < 1 || s.grid * s.threads > (int64_t)UINT32_MAX) say(a, "threads");
  for (const Q8Kernel& o : kQ8Kernels)
    if (q8_shape(a, o).fits() && q8_time(o, a) < q8_time(*k, a)) say(a, "a faster kernel");
  const int64_t cols = k->x_tiles ? 16 * k->x_tiles : q8_tile_x(k->tile);
  const int64_t slots = sorted ? most_tiles(rows, experts, cols) : (rows + cols - 1) / cols;
  if (k->x_tiles) {
    if (s.all_tiles * s.waves * 16 < a.out_rows || s.tiles << s.spread < s.all_tiles) say(a, "tiles");
    if (s.grid < (s.tiles << s.spread) * slots) say(a, "slots");
    if (s.threads != ((k->x_tiles >= 4 && s.waves == 8) ? 512 : 256)) say(a, "waves");
  } else {
    if (s.tiles * q8_tile_w(k->tile) / (glu ? 2 : 1) < a.out_rows) say(a, "tiles");
    if (s.grid < s.tiles * slots || s.grid % 4) say(a, "slots");
  }
}

int main() {
  // Beyond 2^23 workgroups of 512 threads in the kernel that is fastest: 2^29 rows on a few columns, one row on 2^29.
  for (int64_t M : {2, 4, 16})
    for (int64_t K : {1, 100, 128}) {
      check(M, K, (int64_t)1 << 29, 1, false, false);
      check(M, K, (int64_t)1 << 29, 1, false, true);
      check(M, K, (int64_t)1 << 29, 3, true, false);
    }
  for (int64_t M : {(int64_t)1 << 28, (int64_t)1 << 29, (int64_t)1 << 30})
    for (int64_t rows : {1, 2, 17, 64, 65, 130, 300})
      for (bool glu : {false, true}) {
        check(M, 64, rows, 1, false, glu);
        check(M, 64, rows, 1, true, glu);
      }
  std::mt19937_64 rng(1);
  auto log_size = [&](int64_t most) {
    return (int64_t)std::exp(std::uniform_real_distribution<double>(0, std::log((double)most + 0.99))(rng));
  };
  for (int i = 0; i < 200000; ++i) {
    const bool sorted = rng() & 1;
    check(log_size(1 << 30), log_size(1 << 17), log_size(INT32_MAX), sorted ? (int32_t)log_size(512) : 1, sorted, rng() & 1);
  }
  // Sizes that every kernel's launch holds.
  for (int i = 0; i < 20000; ++i) {
    const int64_t M = log_size(70000), rows = log_size(70000);
    const Q8Call a{M, M, q8_pitch(log_size(1 << 17)), (uint32_t)rows, 1, false, false};
    for (const Q8Kernel& k : kQ8Kernels)
      if (!q8_shape(a, k).fits()) say(a, "refused");
    ++cases;
  }
  std::printf("cases=%d bad=%d\n", cases, bad);
  return bad != 0;
}
