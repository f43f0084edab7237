// How the linear layer's products are cut into tiles: host code by itself.
#pragma once
#include <stdint.h>

namespace mdet {

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Few rows: W is read once.  Beyond 8192 rows of W a split sum over tiles is as fast for one row (16384 x 4096 bf16 22.3 us,
// 23.7 this way) and faster for sixteen (23.4, 32.2), as it is for more rows at any size (17 rows of 4096 x 4096 11.5 us).
inline bool few_rows(int64_t rows, int64_t cols) { return rows <= 16 && cols <= 8192; }

// How a product is cut: tile shape and parts of the sum over k.
struct Cut {
  int tile;                            // rows and columns of a tile: 32, 64, 128 or 256; 0: few rows
  int splits;
  int64_t kpart;
};
inline Cut cut_of(int64_t rows, int64_t cols, int64_t k, int64_t size, bool inner) {
  Cut c;
  if (inner && few_rows(rows, cols)) return Cut{0, 1, k};
  const int64_t bk = 128 / size;
  auto tiles = [&](int64_t b) { return ceil_div(rows, b) * ceil_div(cols, b); };
  // The largest tile with which the device is full.  In 16 bits larger tiles also need less of LDS and cache for a product
  // (2500^3, 400 tiles of 128: 59 us, 80 with 64; 2048^3, 256 of them: 28 and 27, k outer 34 and 29); in fp32 the matrix
  // cores are slow enough for the small tile, whose workgroups even out (2500^3 303 and 266 us, 4096^3 962 us with 128).
  c.tile = size == 2 && tiles(256) >= 192 ? 256 : tiles(128) > (size == 2 ? 256 : 800) ? 128 : tiles(64) >= 256 ? 64 : 32;
  c.splits = 1;
  c.kpart = k;
  const int64_t t = tiles(c.tile);
  if (c.tile == 32 && t > 0 && t < 256 && k >= 8 * bk) {
    int64_t most = k / (4 * bk), want = ceil_div(512, t);
    int64_t s = want < most ? want : most;
    if (s > 16) s = 16;
    if (s > 1) {
      c.kpart = ceil_div(ceil_div(k, s), bk) * bk;
      c.splits = (int)ceil_div(k, c.kpart);
    }
  }
  return c;
}

}  // namespace mdet
