// How the linear layer's products are cut into tiles: host code by itself.
#pragma once
#include <stdint.h>

namespace mdet {

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Few rows of x: a kernel of their own reads W once, in place of tiles, which take the same time for 1 as for 32 rows.  Each with W out of
// memory, for 1, 4 and 16 rows, in us (tiles): bf16 4096 x 4096 8.7, 9.1, 11.0 (11.8); 8192 x 4096 14.1, 14.7, 19.3 (18.2); 16384 x 4096
// 24.7, 25.9, 36 (31); 9000 x 8192 34, 37.6, 51 (36.6); 40000 x 4096 55, 59, 84 (79).  fp32 8192 x 4096 26.7, 27.0, 37 (39); 16384 x 4096
// 50, 50, 70 (123); 40000 x 1024 38, 41, 52 (52).  In 16 bits a 16-row product of a long W is bound by the rows' own loads.
// The last condition keeps a launch below 2^32 threads.
inline bool few_rows(int64_t rows, int64_t cols, int64_t size) {
  return rows <= 16 && (size == 4 || rows <= 4 || cols <= 8192) && cols <= (int64_t(1) << 25);
}

// How a product is cut: tile shape and parts of the sum over k.
struct Cut {
  int tile;                            // rows and columns of a tile: 32, 64, 128 or 256; 0: few rows
  int splits;
  int64_t kpart;
};
inline Cut cut_of(int64_t rows, int64_t cols, int64_t k, int64_t size, bool inner) {
  Cut c;
  if (inner && few_rows(rows, cols, size)) return Cut{0, 1, k};
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
