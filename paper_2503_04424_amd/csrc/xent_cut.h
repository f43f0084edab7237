// How the cross entropy is cut into strips and pieces of the vocabulary, and what its workspaces hold: host code by itself.
#pragma once
#include "linear_cut.h"

namespace mdet {

constexpr int64_t XENT_COPY = 768, XENT_COPY_GRAD = 512;

inline uint64_t xent_up256(uint64_t x) { return (x + 255) / 256 * 256; }

// Elements from row to row of what the library lays out itself: whole pieces of 16 bytes, and lines of 128 where rows are long: a slab's 128 bytes
// would lie in two of them (4096 rows of e over 50003 words: dx 408 us and 357, e from what was kept 203 and 164).
inline int64_t xent_pad(int64_t k) { return k >= 1024 ? ceil_div(k, 64) * 64 : ceil_div(k, 8) * 8; }
// Rows of x and W in 16 bits that are no whole pieces of 16 bytes long go through registers, which halves the rate of a product of large tiles.
// From these many rows of x on they are copied first, with zeros behind them.  us without and with copies, 32003 words of
// 1501 in fp16: forward 512 rows 76 and 85, 1024 rows 144 and 127, 4096 rows 523 and 380; gradient 256 rows 352 and 361, 512 rows 295 and 298
// (131071 words: 1156 and 1103), 4096 rows 1636 and 1266.
// The rule knows the rows' length, which a workspace query is told, not their distance or address.  So rows that are whole pieces long and stand
// off 16 bytes go through registers (4096 rows of 1024 over 50003 words in bf16, forward and gradient: 1027 apart 510 and 1498 us, 1024 apart 368 and
// 1151), and rows that are not, at a distance that is, are copied all the same (1021 long and 1024 apart 404 and 1246; 1021 apart 407 and 1251).
inline bool xent_copies(int64_t m, int64_t k, int64_t size, bool backward) { return size == 2 && k % 8 != 0 && m >= (backward ? XENT_COPY_GRAD : XENT_COPY); }

// m rows, a vocabulary of n, rows of k elements of `size` bytes; kept_size: bytes of an exponential that is kept.
struct XentLayout {
  Cut cut;                             // of the forward pass; its sums are not split
  int64_t strip, across;               // columns of a strip, strips of a row
  int64_t ldexps;
  uint64_t exps_bytes, strips_bytes, picked_bytes;
  bool copies;                         // of x and W, in the workspace
  uint64_t x_bytes, w_bytes;
  uint64_t kept() const { return exps_bytes + strips_bytes + picked_bytes; }
  uint64_t workspace(bool keep) const { return x_bytes + w_bytes + (keep ? 0 : strips_bytes + picked_bytes); }
};
inline XentLayout xent_layout(int64_t m, int64_t n, int64_t k, int64_t size, int64_t kept_size) {
  XentLayout l;
  // a workgroup of 256 threads for 16 columns or more, fewer than 2^32 of all
  l.cut = m <= 16 && n <= (int64_t(1) << 27) ? Cut{0, 1, k} : cut_of(m, n, k, size, false);
  // a wavefront's columns of a tile
  l.strip = l.cut.tile == 256 ? 64 : l.cut.tile == 128 ? 64 : l.cut.tile == 64 ? 32 : 16;
  l.across = ceil_div(n, l.strip);
  l.ldexps = xent_pad(n);
  l.exps_bytes = xent_up256((uint64_t)m * l.ldexps * kept_size);
  l.strips_bytes = xent_up256((uint64_t)m * l.across * 8);
  l.picked_bytes = xent_up256((uint64_t)m * 4);
  l.copies = xent_copies(m, k, size, false);
  l.x_bytes = l.copies ? xent_up256((uint64_t)m * xent_pad(k) * size) : 0;
  l.w_bytes = l.copies ? xent_up256((uint64_t)n * xent_pad(k) * size) : 0;
  return l;
}

// Columns of the vocabulary that the gradient takes at once: e has 2^29 elements at most (1 GiB in 16 bits), so long as that leaves
// pieces of 4096; dx adds the pieces up in fp32, which costs a piece of 4096 about 8 % of its products' time.
inline int64_t xent_piece(int64_t m, int64_t n) {
  int64_t most = m > 0 ? (int64_t(1) << 29) / m / 256 * 256 : n;
  if (most < 4096) most = 4096;
  const int64_t pieces = ceil_div(n, most);
  return pieces <= 1 ? n : ceil_div(ceil_div(n, pieces), 256) * 256;
}

// How a product with e is shared out.
struct XentCut {
  int tile;                            // rows and columns of a tile
  int64_t down, across, whole;         // tiles, and how many of them are one workgroup's
  int splits;                          // workgroups of each of the others
  int64_t kpart;
  int64_t units() const { return whole + splits * (down * across - whole); }
  uint64_t bytes() const { return splits > 1 ? xent_up256((uint64_t)(units() - whole) * tile * tile * 4) : 0; }
};
// Tiles of 256 in 16 bits also where they are few, if sums are long: the tiles behind the last whole round of 256 workgroups are shared by as
// many workgroups each as fill another round, of at least eight slabs each.
inline XentCut xent_cut(int64_t rows, int64_t cols, int64_t k, int64_t size) {
  const Cut c = cut_of(rows, cols, k, size, false);
  XentCut x;
  const int64_t large = ceil_div(rows, 256) * ceil_div(cols, 256), rest = large % 256;
  int64_t splits = rest ? 256 / rest : 1, most = k / 512;
  if (splits > 16) splits = 16;
  if (splits > most) splits = most;
  // a unit of 64 of k is 1.7 us; the parts of a round are written and read in 35
  const bool worth = size == 2 && splits > 1 && (double)k * 0.026 * (1.0 - 1.0 / (double)splits) > 35.0;
  if (worth && (c.tile == 256 || rest * splits >= 160 || large > 256)) {
    x.tile = 256;
    x.whole = large - rest;
    x.splits = (int)splits;
    x.kpart = ceil_div(ceil_div(k, splits), 64) * 64;
    x.splits = (int)ceil_div(k, x.kpart);
  } else {
    x.tile = c.tile;
    x.splits = c.splits;
    x.kpart = c.kpart;
    x.whole = c.splits > 1 ? 0 : ceil_div(rows, c.tile) * ceil_div(cols, c.tile);
  }
  x.down = ceil_div(rows, x.tile);
  x.across = ceil_div(cols, x.tile);
  return x;
}

struct XentGradLayout {
  int64_t piece, lde, ldrows;
  bool copies;                         // of a piece of W; x's is there anyway
  uint64_t e, rows, scale, sums, total, w, parts, bytes;
};
// parts_of_e: numbers of the operands' type that add up to an element of e.
inline XentGradLayout xent_grad_layout(int64_t m, int64_t n, int64_t k, int64_t size, int64_t parts_of_e) {
  XentGradLayout l;
  l.piece = xent_piece(parts_of_e * m, n);
  l.lde = xent_pad(l.piece);
  l.ldrows = xent_pad(k);
  l.copies = xent_copies(m, k, size, true);
  l.e = 0;
  l.rows = xent_up256((uint64_t)parts_of_e * m * l.lde * size);
  l.scale = l.rows + xent_up256((uint64_t)parts_of_e * m * l.ldrows * size);
  l.sums = l.scale + 256;
  // column sums of strips of 16 rows or more, of whole tiles
  l.total = l.sums + xent_up256((uint64_t)(ceil_div(m, 256) * 16) * l.piece * 4);
  l.w = l.total + (l.piece < n ? xent_up256((uint64_t)m * k * 4) : 0);
  l.parts = l.w + (l.copies ? xent_up256((uint64_t)l.piece * l.ldrows * size) : 0);
  uint64_t parts = 0;
  auto room = [&](int64_t rows, int64_t cols, int64_t inner) {
    const uint64_t b = xent_cut(rows, cols, inner, size).bytes();
    if (b > parts) parts = b;
  };
  const int64_t last = n > 0 ? n - (n - 1) / l.piece * l.piece : 0;
  room(m, k, l.piece);
  room(m, k, last);
  room(l.piece, k, parts_of_e * m);
  room(last, k, parts_of_e * m);
  l.bytes = l.parts + parts;
  return l;
}

}  // namespace mdet
