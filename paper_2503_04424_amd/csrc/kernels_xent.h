// Softmax cross entropy of a linear layer over a large vocabulary, and its gradient, without its logits in memory.
//
//   z = x W^T + b;  lse_i = log(sum over j of exp(z_ij));  loss_i = lse_i - z_i,t_i
//   e_ij = g_i (exp(z_ij - lse_i) - [j = t_i]);  dx = e W;  dW = e^T x;  db = column sums of e
//
// Forward, each tile of z stays in the accumulators: what leaves it are each row's largest logit M and the sum of exp(z - M) over the
// tile's columns (a strip), joined by a second launch, and the logit of the target.  Backward, z is formed once more in front
// of e, a piece of the vocabulary at a time; or, where the forward pass kept them, exp(z - M) is read back in the operands' type (M is the
// strip's: nothing overflows, and what is rounded keeps its relative precision), which spares that product.
//
// Sums and everything behind them are fp32; e is rounded to the operands' type in front of its two products, db sums the unrounded one.
// In fp16 e would vanish below 2^-24, where most probabilities of a large vocabulary lie: it is scaled by a power of two
// that brings the largest |g| to 2^14 .. 2^15, and the products by its reciprocal.
//
// Rows whose target lies outside of the vocabulary, or is `ignore`, do not count: loss 0, e exactly 0 whatever their logits are, and zeros
// in the place of their x in dW, so that nothing of them comes through.
#pragma once
#include "kernels_linear.h"
#include "kernels_rows.h"

namespace mdet {

struct XentTargets {
  const void* target;
  int bits;                            // 32 or 64
  int64_t ignore, vocab;
};
// The target of row i; -1 if it does not count.
__device__ __forceinline__ int64_t xent_target(const XentTargets& t, const int64_t i) {
  const int64_t v = t.bits == 32 ? (int64_t) static_cast<const int32_t*>(t.target)[i] : static_cast<const int64_t*>(t.target)[i];
  return v < 0 || v >= t.vocab || v == t.ignore ? -1 : v;
}

// exp(z - top) where top is the largest of some z: zero for z = -inf also where that is all there is.
__device__ __forceinline__ float xent_exp(const float z, const float top) {
  return __expf(z - (top == -INFINITY ? 0.0f : top));
}

struct XentStrip {                     // of a row: its largest logit among a strip's columns, and the sum of exp(z - top)
  float top, sum;
};

template <typename T>
struct XentForward {
  XentTargets t;
  const T* bias;                       // null: none
  XentStrip* strips;                   // rows x across
  int64_t across;
  float* picked;                       // of the rows that count: the target's logit
  T* exps;                             // rows x ldexps, exp(z - top); null: not kept
  int64_t ldexps, rows, cols;
};

// A tile: its logits, then what is left of each of its rows.
template <typename T, typename S, bool DIRECT>
__global__ __launch_bounds__(S::THREADS) void xent_forward_kernel(const Operand<T> r, const Operand<T> c, const int64_t k, const XentForward<T> o,
                                                                  const int64_t tiles) {
  typedef typename Core<T>::acc_t acc_t;
  constexpr int ROWS = S::TM * 16;
  __shared__ __attribute__((aligned(16))) char lds[LinearLds<S>::BYTES];
  const int64_t t = gemm_tile_number(blockIdx.x, tiles);
  if (t < 0) return;
  int64_t bi, bj;
  gemm_tile_place(t, (o.rows + S::BM - 1) / S::BM, o.across, bi, bj);
  const int64_t row0 = bi * S::BM, col0 = bj * S::BN;
  acc_t acc[S::TN][S::TM] = {};
  TileStream<T, S, false, false, DIRECT> stream(lds);
  auto none = [] { return false; };
  stream.set(r, c, row0, col0, 0, k);
  stream.begin(none);
  stream.run(acc, stream.slabs(0, k), none);

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int64_t wrow = row0 + wave / S::WN * ROWS, wcol = col0 + wave % S::WN * (S::TN * 16) + 4 * (lane >> 4);
#pragma unroll
  for (int a = 0; a < S::TN; ++a)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t j = wcol + 16 * a + e;
      const bool there = j < o.cols;
      const float add = o.bias && there ? (float)o.bias[j] : 0.0f;
#pragma unroll
      for (int b = 0; b < S::TM; ++b) acc[a][b][e] = there ? acc[a][b][e] + add : -INFINITY;
    }
  // the rows' largest: of this wavefront, then of those beside it
  __syncthreads();                     // the operands are not read any more
  float* const tops = reinterpret_cast<float*>(lds);           // of each wavefront's rows
  float* const sums = tops + S::WAVES * ROWS;
  auto beside = [&](float* const of, const int row, auto&& f) {
#pragma unroll
    for (int w = 0; w < S::WN; ++w) f(of[(wave / S::WN * S::WN + w) * ROWS + row]);
  };
#pragma unroll
  for (int b = 0; b < S::TM; ++b) {
    float m = -INFINITY;
#pragma unroll
    for (int a = 0; a < S::TN; ++a)
#pragma unroll
      for (int e = 0; e < 4; ++e) m = fmaxf(m, acc[a][b][e]);
    m = fmaxf(m, __shfl_xor(m, 16, 64));
    m = fmaxf(m, __shfl_xor(m, 32, 64));
    if (lane < 16) tops[wave * ROWS + 16 * b + lane] = m;
  }
  __syncthreads();
#pragma unroll
  for (int b = 0; b < S::TM; ++b) {
    const int row = 16 * b + (lane & 15);
    const int64_t i = wrow + row;
    float top = -INFINITY;
    beside(tops, row, [&](const float v) { top = fmaxf(top, v); });
    const int64_t target = i < o.rows ? xent_target(o.t, i) : -1;
    const int at = target >= wcol && target < wcol + S::TN * 16 ? (int)(target - wcol) : -1;
    float s = 0.0f;
#pragma unroll
    for (int a = 0; a < S::TN; ++a)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (at == 16 * a + e) o.picked[i] = acc[a][b][e];
        acc[a][b][e] = xent_exp(acc[a][b][e], top);
        s += acc[a][b][e];
      }
    s += __shfl_xor(s, 16, 64);
    s += __shfl_xor(s, 32, 64);
    if (lane < 16) sums[wave * ROWS + 16 * b + lane] = s;
  }
  __syncthreads();
  if (wave % S::WN == 0)
    for (int row = lane; row < ROWS; row += 64) {
      const int64_t i = wrow + row;
      XentStrip x{-INFINITY, 0.0f};
      beside(tops, row, [&](const float v) { x.top = fmaxf(x.top, v); });
      beside(sums, row, [&](const float v) { x.sum += v; });
      if (i < o.rows) o.strips[i * o.across + bj] = x;
    }
  if (!o.exps) return;
  __syncthreads();
  tile_rows<T, S>(lds, acc, row0, col0, o.rows, o.cols, [&](auto&& rows) {
    rows([&](const int64_t i, const int64_t j, const float (&in)[4]) {
      typedef T t4 __attribute__((ext_vector_type(4)));
      // rows are ceil(cols / 8) 8 long: what is written behind their end is zero
      *reinterpret_cast<t4*>(o.exps + i * o.ldexps + j) = t4{(T)in[0], (T)in[1], (T)in[2], (T)in[3]};
    });
  });
}

// Up to 16 rows: W is read once, 16 rows of it, a strip, by a workgroup.
template <typename T, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void xent_forward_rows_kernel(const Operand<T> x, const Operand<T> w, const int64_t k, const XentForward<T> o) {
  const int lane = threadIdx.x & 63, i = lane & 15;
  const int64_t col0 = (int64_t)blockIdx.x * 16, c = col0 + 4 * (lane >> 4);
  const typename Core<T>::acc_t sum = linear_rows_sum<T, WAVES>(x, w, k, col0);
  if (threadIdx.x >= 64) return;
  const int64_t target = i < o.rows ? xent_target(o.t, i) : -1;
  float z[4], top = -INFINITY, s = 0.0f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    z[e] = c + e < o.cols ? sum[e] + (o.bias ? (float)o.bias[c + e] : 0.0f) : -INFINITY;
    top = fmaxf(top, z[e]);
    if (c + e == target) o.picked[i] = z[e];
  }
  top = fmaxf(top, __shfl_xor(top, 16, 64));
  top = fmaxf(top, __shfl_xor(top, 32, 64));
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    z[e] = xent_exp(z[e], top);
    s += z[e];
  }
  s += __shfl_xor(s, 16, 64);
  s += __shfl_xor(s, 32, 64);
  if (i >= o.rows) return;
  if (lane < 16) o.strips[i * o.across + blockIdx.x] = XentStrip{top, s};
  typedef T t4 __attribute__((ext_vector_type(4)));
  if (o.exps && c < o.cols) *reinterpret_cast<t4*>(o.exps + i * o.ldexps + c) = t4{(T)z[0], (T)z[1], (T)z[2], (T)z[3]};
}

// lse and loss of a row from its strips, by LANES lanes.
template <int LANES>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void xent_join_kernel(const XentStrip* __restrict__ strips, const int64_t across,
                                                                              const float* __restrict__ picked, const XentTargets t, const int64_t rows,
                                                                              float* __restrict__ loss, float* __restrict__ lse, const int64_t first) {
  constexpr int THREADS = LANES < 256 ? 256 : LANES, WAVES = THREADS / 64;
  __shared__ XentStrip part[WAVES];
  const int64_t row = (first + blockIdx.x) * (THREADS / LANES) + threadIdx.x / LANES;
  if (row >= rows) return;             // whole wavefronts, or the whole workgroup
  XentStrip all{-INFINITY, 0.0f};
  auto add = [&](const XentStrip& s) {
    const float top = fmaxf(all.top, s.top);
    all.sum = all.sum * xent_exp(all.top, top) + s.sum * xent_exp(s.top, top);
    all.top = top;
  };
  for (int64_t s = threadIdx.x % LANES; s < across; s += LANES) add(strips[row * across + s]);
#pragma unroll
  for (int off = 1; off < 64; off *= 2) add(XentStrip{__shfl_xor(all.top, off, 64), __shfl_xor(all.sum, off, 64)});
  if constexpr (LANES > 64) {
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = all;
    __syncthreads();
    all = part[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) add(part[w]);
  }
  if (threadIdx.x % LANES == 0) {
    const float l = all.top + logf(all.sum);
    if (lse) lse[row] = l;
    if (loss) loss[row] = xent_target(t, row) >= 0 ? l - picked[row] : 0.0f;
  }
}

// ---------------------------------------------------------------------------
// The gradient.
// ---------------------------------------------------------------------------

// Powers of two: what e is scaled by, and its reciprocal.
struct XentScale {
  float up, down;
};

// For operands in fp16: the largest |g| of a row that counts comes to 2^14 .. 2^15.
__global__ __launch_bounds__(1024) void xent_scale_kernel(const float* __restrict__ g, const XentTargets t, const int64_t rows, XentScale* scale) {
  __shared__ float part[16];
  float most = 0.0f;
  for (int64_t i = threadIdx.x; i < rows; i += 1024)
    if (xent_target(t, i) >= 0) most = fmaxf(most, fabsf(g[i]));
#pragma unroll
  for (int off = 1; off < 64; off *= 2) most = fmaxf(most, __shfl_xor(most, off, 64));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = most;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 16; ++w) most = fmaxf(most, part[w]);
    int up = 0;
    if (most > 0.0f && most < INFINITY) up = 14 - ilogbf(most);
    up = up > 120 ? 120 : up < -100 ? -100 : up;
    *scale = XentScale{ldexpf(1.0f, up), ldexpf(1.0f, -up)};
  }
}

// x with zeros in the rows that do not count, rows on 16 bytes.
template <typename T>
__global__ __launch_bounds__(256) void xent_rows_kernel(const T* __restrict__ x, const int64_t ldx, const XentTargets t, const int64_t rows,
                                                        const int64_t k, T* __restrict__ to, const int64_t ldto, const int64_t first) {
  typedef typename Core<T>::piece_t piece_t;
  const int64_t across = ldto / Core<T>::VEC, id = (first + blockIdx.x) * 256 + threadIdx.x, i = id / across, c = (id - i * across) * Core<T>::VEC;
  if (i >= rows) return;
  piece_t v = {};
  if (xent_target(t, i) >= 0) v = row_piece<T>(x + i * ldx, c, k);
  *reinterpret_cast<piece_t*>(to + i * ldto + c) = v;
}

template <typename T>
struct XentSlope {
  XentTargets t;
  const T* bias;                       // null: none
  const float *lse, *g;
  const XentScale* scale;              // null: 1
  T* e;                                // rows x lde, columns from `first` on
  int64_t lde;
  float* sums;                         // parts x cols of db; null: not wanted
  int64_t rows, cols, first;           // of the piece
};

// What a row needs for its e: its weight (zero if it does not count), its target, counted from column `from` on.
struct XentRow {
  float lse, g;
  bool counts;
  int64_t target;
};
template <typename T>
__device__ __forceinline__ XentRow xent_row(const XentSlope<T>& o, const int64_t i, const int64_t from) {
  XentRow r{0.0f, 0.0f, false, -1};
  if (i >= o.rows) return r;
  const int64_t t = xent_target(o.t, i);
  if (t < 0) return r;
  return XentRow{o.lse[i], o.g[i], true, t - o.first - from};
}

// A tile of e.
template <typename T, typename S, bool DIRECT>
__global__ __launch_bounds__(S::THREADS) void xent_slope_kernel(const Operand<T> r, const Operand<T> c, const int64_t k, const XentSlope<T> o,
                                                                const int64_t tiles) {
  typedef typename Core<T>::acc_t acc_t;
  constexpr int ROWS = S::TM * 16;
  __shared__ __attribute__((aligned(16))) char lds[LinearLds<S>::BYTES];
  const int64_t t = gemm_tile_number(blockIdx.x, tiles);
  if (t < 0) return;
  int64_t bi, bj;
  gemm_tile_place(t, (o.rows + S::BM - 1) / S::BM, (o.cols + S::BN - 1) / S::BN, bi, bj);
  const int64_t row0 = bi * S::BM, col0 = bj * S::BN;
  acc_t acc[S::TN][S::TM] = {};
  TileStream<T, S, false, false, DIRECT> stream(lds);
  auto none = [] { return false; };
  stream.set(r, c, row0, col0, 0, k);
  stream.begin(none);
  stream.run(acc, stream.slabs(0, k), none);

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int64_t wrow = row0 + wave / S::WN * ROWS, wcol = col0 + wave % S::WN * (S::TN * 16) + 4 * (lane >> 4);
  const float up = o.scale ? o.scale->up : 1.0f;
  float add[S::TN][4], sum[S::TN][4] = {};
#pragma unroll
  for (int a = 0; a < S::TN; ++a)
#pragma unroll
    for (int e = 0; e < 4; ++e) add[a][e] = o.bias && wcol + 16 * a + e < o.cols ? (float)o.bias[wcol + 16 * a + e] : 0.0f;
#pragma unroll
  for (int b = 0; b < S::TM; ++b) {
    const XentRow row = xent_row(o, wrow + 16 * b + (lane & 15), wcol);
    const int at = row.target >= 0 && row.target < S::TN * 16 ? (int)row.target : -1;
#pragma unroll
    for (int a = 0; a < S::TN; ++a)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p = __expf(acc[a][b][e] + add[a][e] - row.lse);
        const float v = row.counts ? (at == 16 * a + e ? p - 1.0f : p) * row.g : 0.0f;
        sum[a][e] += v;
        acc[a][b][e] = v * up;
      }
  }
  if (o.sums) {
    const int64_t part = bi * S::WM + wave / S::WN;
#pragma unroll
    for (int a = 0; a < S::TN; ++a)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float s = sum[a][e];
#pragma unroll
        for (int off = 1; off < 16; off *= 2) s += __shfl_xor(s, off, 64);
        const int64_t j = wcol + 16 * a + e;
        if ((lane & 15) == 0 && j < o.cols) o.sums[part * o.cols + j] = s;
      }
  }
  __syncthreads();                     // the operands are not read any more
  tile_rows<T, S>(lds, acc, row0, col0, o.rows, o.cols, [&](auto&& rows) {
    rows([&](const int64_t i, const int64_t j, const float (&in)[4]) {
      typedef T t4 __attribute__((ext_vector_type(4)));
      // rows of e are whole pieces of 16 bytes long
      *reinterpret_cast<t4*>(o.e + i * o.lde + j) = t4{(T)in[0], (T)in[1], (T)in[2], (T)in[3]};
    });
  });
}

// e from what the forward pass kept: 16 EACH rows of 16 pieces by a workgroup, as in the gradient of the activation.
constexpr int XENT_EACH = 4;

template <typename T>
__global__ __launch_bounds__(256) void xent_slope_kept_kernel(const XentSlope<T> o, const T* __restrict__ exps, const int64_t ldexps,
                                                              const XentStrip* __restrict__ strips, const int64_t across, const int64_t strip,
                                                              const float* __restrict__ picked, const int64_t first) {
  typedef typename Core<T>::piece_t piece_t;
  constexpr int VEC = Core<T>::VEC;
  __shared__ float part[16][16 * VEC];
  const int64_t wide = (o.cols + 16 * VEC - 1) / (16 * VEC), id = first + blockIdx.x, down = id / wide;
  const int t = threadIdx.x / 16, c = threadIdx.x % 16 * VEC;
  const int64_t col0 = (id - down * wide) * (16 * VEC), col = col0 + c, row = down * (16 * XENT_EACH) + t;
  const bool there = col < o.cols;
  const float up = o.scale ? o.scale->up : 1.0f;
  piece_t x[XENT_EACH];
  XentRow of[XENT_EACH];
  float top[XENT_EACH], hit[XENT_EACH];
#pragma unroll
  for (int r = 0; r < XENT_EACH; ++r) {
    const int64_t i = row + 16 * r;
    of[r] = xent_row(o, i, col);
    x[r] = piece_t{};
    top[r] = hit[r] = 0.0f;
    if (of[r].counts && there) {
      x[r] = *reinterpret_cast<const piece_t*>(exps + i * ldexps + o.first + col);
      top[r] = strips[i * across + (o.first + col) / strip].top;
      hit[r] = picked[i];
    }
  }
  float sum[VEC] = {};
#pragma unroll
  for (int r = 0; r < XENT_EACH; ++r) {
    const int64_t i = row + 16 * r;
    // the strip may hold nothing but -inf, beside a row's finite logits
    const float share = top[r] == -INFINITY ? __expf(-of[r].lse) : __expf(top[r] - of[r].lse);
    piece_t d;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float p = (float)x[r][e] * share;
      // the target's own from its logit: a probability near 1 loses what is left of it in 16 bits
      const float q = of[r].target == e ? __expf(hit[r] - of[r].lse) - 1.0f : p;
      const float v = of[r].counts ? q * of[r].g : 0.0f;
      if (i < o.rows) sum[e] += v;
      d[e] = (T)(v * up);
    }
    if (i < o.rows && there) *reinterpret_cast<piece_t*>(o.e + i * o.lde + col) = d;
  }
  if (!o.sums) return;
#pragma unroll
  for (int e = 0; e < VEC; ++e) part[t][c + e] = sum[e];
  __syncthreads();
  if (threadIdx.x < 16 * VEC && col0 + threadIdx.x < o.cols) {
    float v = part[0][threadIdx.x];
#pragma unroll
    for (int r = 1; r < 16; ++r) v += part[r][threadIdx.x];
    o.sums[down * o.cols + col0 + threadIdx.x] = v;
  }
}

// db of a piece: its parts, added in one order, sixteen threads a column.
template <typename O>
__global__ __launch_bounds__(256) void xent_columns_kernel(const float* __restrict__ sums, const int64_t parts, const int64_t cols, O* __restrict__ db,
                                                           const int64_t first) {
  __shared__ float part[16][16];
  const int t = threadIdx.x / 16, c = threadIdx.x % 16;
  const int64_t col = (first + blockIdx.x) * 16 + c;
  float sum = 0.0f;
  if (col < cols)
    for (int64_t s = t; s < parts; s += 16) sum += sums[s * cols + col];
  part[t][c] = sum;
  __syncthreads();
  if (t == 0 && col < cols) {
    float v = part[0][c];
#pragma unroll
    for (int r = 1; r < 16; ++r) v += part[r][c];
    db[col] = (O)v;
  }
}

// Where a product with e goes: y, or, for dx over several pieces of the vocabulary, the sum over those so far.
template <typename O>
struct XentOut {
  O* y;
  int64_t ldy;
  const XentScale* scale;              // null: 1
  float* total;                        // rows x cols
  bool begins, ends;                   // the first, the last piece
  int64_t rows, cols;
  bool vec;                            // rows of y and total start where four elements can be moved at once
};

template <typename O>
__device__ __forceinline__ void xent_put4(const XentOut<O>& o, const int64_t i, const int64_t j, const float (&in)[4]) {
  typedef O o4 __attribute__((ext_vector_type(4)));
  typedef float f4 __attribute__((ext_vector_type(4)));
  const float down = o.scale ? o.scale->down : 1.0f;
  float* const total = o.total + i * o.cols + j;
  O* const y = o.y + i * o.ldy + j;
  if (o.vec && j + 4 <= o.cols) {
    f4 v = f4{in[0], in[1], in[2], in[3]} * down;
    if (!o.begins) v += *reinterpret_cast<const f4*>(total);
    if (o.ends) *reinterpret_cast<o4*>(y) = o4{(O)v[0], (O)v[1], (O)v[2], (O)v[3]};
    else *reinterpret_cast<f4*>(total) = v;
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (j + e >= o.cols) break;
    const float v = in[e] * down + (o.begins ? 0.0f : total[e]);
    if (o.ends) y[e] = (O)v;
    else total[e] = v;
  }
}

// dx = e W (C outer) and dW = e^T x (both outer).  SPLIT: part t / tiles of the sum over k.
template <typename T, typename O, typename S, bool ROUTER, bool DIRECT, bool SPLIT>
__global__ __launch_bounds__(S::THREADS) void xent_product_kernel(const Operand<T> r, const Operand<T> c, const int64_t k, const XentOut<O> o,
                                                                  const int64_t tiles, float* const parts, const int64_t kpart) {
  __shared__ __attribute__((aligned(16))) char lds[LinearLds<S>::BYTES];
  const int64_t t = gemm_tile_number(blockIdx.x, tiles);
  if (t < 0) return;
  const int64_t down = (o.rows + S::BM - 1) / S::BM, across = (o.cols + S::BN - 1) / S::BN, one = down * across;
  int64_t bi, bj;
  gemm_tile_place(t % one, down, across, bi, bj);
  const int64_t part = t / one, k0 = part * kpart, kend = k0 + kpart < k ? k0 + kpart : k;
  const int64_t row0 = bi * S::BM, col0 = bj * S::BN;
  typename Core<T>::acc_t acc[S::TN][S::TM] = {};
  TileStream<T, S, ROUTER, true, DIRECT> stream(lds);
  auto none = [] { return false; };
  stream.set(r, c, row0, col0, k0, kend);
  stream.begin(none);
  stream.run(acc, stream.slabs(k0, kend), none);
  __syncthreads();                     // the operands are not read any more
  tile_rows<T, S>(lds, acc, row0, col0, o.rows, o.cols, [&](auto&& rows) {
    rows([&](const int64_t i, const int64_t j, const float (&in)[4]) {
      if constexpr (SPLIT) {
        float* const to = parts + (part * o.rows + i) * o.cols + j;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (j + e < o.cols) to[e] = in[e];
      } else xent_put4(o, i, j, in);
    });
  });
}

// The parts of the sum over k, added in their order.
template <typename O>
__global__ __launch_bounds__(256) void xent_product_join_kernel(const float* __restrict__ parts, const int splits, const XentOut<O> o) {
  const int64_t across = (o.cols + 3) / 4, id = (int64_t)blockIdx.x * 256 + threadIdx.x, i = id / across, j = (id - i * across) * 4;
  if (i >= o.rows) return;
  float v[4] = {};
  for (int s = 0; s < splits; ++s)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (j + e < o.cols) v[e] += parts[(s * o.rows + i) * o.cols + j + e];
  xent_put4(o, i, j, v);
}

}  // namespace mdet
