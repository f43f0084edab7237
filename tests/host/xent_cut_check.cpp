// Checks of how the cross entropy is cut, over many sizes: prints the first that fails.
#include <cstdio>
#include <cstdint>
#include <cstdlib>
#include <initializer_list>

#include "../../paper_2503_04424_amd/csrc/xent_cut.h"

using namespace mdet;

#define HOLDS(what)                                                                                                   \
  if (!(what)) {                                                                                                      \
    std::printf("%s: m %lld n %lld k %lld size %d\n", #what, (long long)m, (long long)n, (long long)k, (int)size); \
    return false;                                                                                                     \
  }

static bool cut_holds(int64_t m, int64_t n, int64_t k, int64_t size) {
  const XentCut c = xent_cut(m, n, k, size);
  HOLDS(c.tile == 32 || c.tile == 64 || c.tile == 128 || (c.tile == 256 && size == 2));
  HOLDS(c.down * c.tile >= m && (c.down - 1) * c.tile < m && c.across * c.tile >= n && (c.across - 1) * c.tile < n);
  HOLDS(c.whole >= 0 && c.whole <= c.down * c.across && c.splits >= 1 && c.splits <= 16);
  // the parts of a sum: none of them empty, none left out; one part is the whole
  HOLDS(c.splits == 1 ? c.kpart >= k : c.kpart * (c.splits - 1) < k && c.kpart * c.splits >= k && c.kpart % (128 / size) == 0);
  HOLDS(c.splits > 1 || c.units() == c.down * c.across);
  HOLDS(c.splits == 1 || c.bytes() >= (uint64_t)(c.down * c.across - c.whole) * c.splits * c.tile * c.tile * 4);
  HOLDS(c.units() < (int64_t(1) << 31));
  return true;
}

static bool holds(int64_t m, int64_t n, int64_t k, int64_t size, int64_t parts) {
  const XentLayout f = xent_layout(m, n, k, size, size);
  HOLDS(f.exps_bytes >= (uint64_t)m * n * size && xent_layout(m, n, k, size, 4).exps_bytes >= (uint64_t)m * n * 4);
  HOLDS(f.across * f.strip >= n && (f.across - 1) * f.strip < n && f.ldexps >= n && f.ldexps % 8 == 0);
  // a wavefront's columns: four of them beside each other in the largest tile, two in the others, one strip of 16 a wavefront for few rows
  HOLDS(f.cut.tile == 256 ? f.strip == 64 : f.cut.tile ? f.strip * 2 == f.cut.tile : f.strip == 16 && m <= 16);
  // a launch is of fewer than 2^32 threads: a workgroup of 256 for 16 columns or more
  HOLDS(f.cut.tile != 0 || ceil_div(n, 16) * 256 < (int64_t(1) << 32));
  const XentGradLayout g = xent_grad_layout(m, n, k, size, parts);
  HOLDS(g.piece >= 1 && g.piece <= n && (g.piece == n || g.piece % 256 == 0) && g.lde >= g.piece && g.lde % 8 == 0 && g.ldrows >= k);
  HOLDS(g.piece == n || parts * m * g.piece <= (int64_t(1) << 29) || g.piece <= 4096);
  HOLDS(g.rows - g.e >= (uint64_t)parts * m * g.lde * size && g.scale - g.rows >= (uint64_t)parts * m * g.ldrows * size && g.sums - g.scale >= 8);
  // column sums: of a tile's wavefronts beneath each other, or of 64 rows
  for (int64_t v = 0; v < n; v += g.piece) {
    const int64_t w = n - v < g.piece ? n - v : g.piece;
    const int tile = cut_of(m, w, k, size, false).tile;
    HOLDS(g.total - g.sums >= (uint64_t)ceil_div(m, tile) * 2 * w * 4 && g.total - g.sums >= (uint64_t)ceil_div(m, 64) * w * 4);
    HOLDS(g.bytes - g.parts >= xent_cut(m, k, w, size).bytes() && g.bytes - g.parts >= xent_cut(w, k, parts * m, size).bytes());
    if (!cut_holds(m, k, w, size) || !cut_holds(w, k, parts * m, size)) return false;
    if (v > 0 && v + 2 * g.piece < n) v = (n - v) / g.piece * g.piece + v - 2 * g.piece;      // pieces between are alike
  }
  HOLDS(g.piece == n || g.w - g.total >= (uint64_t)m * k * 4);
  HOLDS(!g.copies || (size == 2 && k % 8 != 0 && g.parts - g.w >= (uint64_t)g.piece * g.ldrows * size && g.ldrows % 8 == 0));
  HOLDS(!f.copies || (size == 2 && k % 8 != 0 && f.x_bytes >= (uint64_t)m * xent_pad(k) * size && f.w_bytes >= (uint64_t)n * xent_pad(k) * size));
  HOLDS(xent_pad(k) >= k && xent_pad(k) % 8 == 0);
  return true;
}

// A vocabulary of 2^28 words, and a few more or less, for one row and for sixteen.
static bool launches_hold() {
  for (int64_t m = 1; m <= 16; m += 15)
    for (int64_t n = (int64_t(1) << 27) - 1; n < (int64_t(1) << 28) + 64; n = n < (int64_t(1) << 27) + 2 || n >= (int64_t(1) << 28) - 64 ? n + 1 : (int64_t(1) << 28) - 64) {
      const int64_t k = 1, size = 2;
      HOLDS(xent_layout(m, n, k, size, size).cut.tile != 0 || ceil_div(n, 16) * 256 < (int64_t(1) << 32));
    }
  return true;
}

int main() {
  if (!launches_hold()) return 1;
  const int64_t sizes[] = {1, 2, 15, 16, 17, 33, 64, 65, 100, 127, 129, 255, 256, 257, 300, 512, 777, 1000, 1024, 1500, 2048, 4096, 5003, 8192, 9000, 16384, 32000,
                           50003, 65536, 131072, 140000, 1000000};
  for (const int64_t m : sizes)
    for (const int64_t n : sizes)
      for (const int64_t k : sizes)
        for (const int64_t size : {int64_t(2), int64_t(4)})
          if (m * n <= (int64_t(1) << 36) && n * k <= (int64_t(1) << 36) && m * k <= (int64_t(1) << 36))
            for (int64_t parts = 1; parts <= (size == 2 ? 3 : 1); ++parts)
              if (!holds(m, n, k, size, parts)) return 1;
  std::srand(1);
  for (int i = 0; i < 200000; ++i) {
    const int64_t m = 1 + std::rand() % 9000, n = 1 + std::rand() % 140000, k = 1 + std::rand() % 9000;
    if (!holds(m, n, k, i % 2 ? 2 : 4, i % 2 ? 1 + i / 2 % 3 : 1)) return 1;
  }
  return 0;
}
