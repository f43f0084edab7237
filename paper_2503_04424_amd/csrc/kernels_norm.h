// Layer norm over the rows of a matrix, and its gradient.
//
//   mean = avg(x), var = avg((x - mean)^2), rstd = 1 / sqrt(var + eps);  h = (x - mean) rstd;  y = h w + b
//   u = dy w;  dx = rstd (u - avg(u) - h avg(u h));  dw = column sums of dy h, db those of dy
//
// Everything is fp32 until the one rounding of what is stored.  The variance is the mean of the squares around the mean, from
// the row in registers: a difference of mean squares would lose what a large mean has over it.
#pragma once
#include "kernels_rows.h"

namespace mdet {

constexpr int NORM_THREADS = 256;

// Sum over the row's lanes, in all of them.
template <int LANES>
__device__ __forceinline__ float norm_lanes_sum(float v) {
#pragma unroll
  for (int off = 1; off < (LANES < 64 ? LANES : 64); off *= 2) v += __shfl_xor(v, off, 64);
  return v;
}

// N sums over the row's lanes, in all of them.  `part` is free again behind the next call's barrier, if that has another one.
template <int LANES, int N>
__device__ __forceinline__ void norm_sums(float (&v)[N], float (*const part)[N]) {
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = norm_lanes_sum<LANES>(v[n]);
  if constexpr (LANES > 64) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int n = 0; n < N; ++n) part[wave][n] = v[n];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {
      float s = part[0][n];
#pragma unroll
      for (int w = 1; w < LANES / 64; ++w) s += part[w][n];
      v[n] = s;
    }
  }
}

template <typename T>
struct NormForward {
  const T* x;
  int64_t ldx;
  const T *w, *b;                      // null: 1 and 0
  T* y;
  int64_t ldy;
  float *mean, *rstd;                  // null: not kept
  int64_t rows, cols;
  float eps, count;                    // cols; a quotient: the mean of equal elements is that element
};

// A row by LANES lanes, P pieces of 16 bytes in each one's registers, so that it is read once for its mean, its variance and its result.  Bytes bound
// it: 16384 x 4096 bf16 45 us (6.0 TB/s, part of it out of the last cache), one row 2.8.
template <typename T, int THREADS, int LANES, int P>
__global__ __launch_bounds__(THREADS) void norm_forward_kernel(const NormForward<T> a, const int64_t first) {
  typedef typename Core<T>::piece_t piece_t;
  constexpr int VEC = Core<T>::VEC;
  __shared__ float part[2][THREADS / 64][1];
  const int lane = threadIdx.x % LANES;
  const int64_t row = (first + blockIdx.x) * (THREADS / LANES) + threadIdx.x / LANES;
  if (row >= a.rows) return;           // whole waves, or parts of one that no sum reaches
  const T* const x = a.x + row * a.ldx;
  piece_t raw[P];
#pragma unroll
  for (int p = 0; p < P; ++p) raw[p] = row_piece<T>(x, (int64_t)(p * LANES + lane) * VEC, a.cols);
  float sum[1] = {0.0f};
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int e = 0; e < VEC; ++e) sum[0] += (float)raw[p][e];
  norm_sums<LANES, 1>(sum, part[0]);
  const float mean = sum[0] / a.count;
  float square[1] = {0.0f};
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float d = (float)raw[p][e] - mean;
      if ((p * LANES + lane) * VEC + e < a.cols) square[0] += d * d;
    }
  norm_sums<LANES, 1>(square, part[1]);
  const float rstd = 1.0f / sqrtf(square[0] / a.count + a.eps);
  if (lane == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
  T* const y = a.y + row * a.ldy;
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int64_t c = (int64_t)(p * LANES + lane) * VEC;
    if (c >= a.cols) break;
    piece_t w, b;
    float out[VEC];
    if (a.w) w = row_piece<T>(a.w, c, a.cols);
    if (a.b) b = row_piece<T>(a.b, c, a.cols);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      float v = ((float)raw[p][e] - mean) * rstd;
      if (a.w) v *= (float)w[e];
      if (a.b) v += (float)b[e];
      out[e] = v;
    }
    row_store<T, T>(y, c, a.cols, out);
  }
}

// Rows that no workgroup has registers for: the row is read three times, the second and third time out of cache.
template <typename T>
__global__ __launch_bounds__(1024) void norm_forward_long_kernel(const NormForward<T> a, const int64_t first) {
  constexpr int VEC = Core<T>::VEC;
  __shared__ float part[2][16][1];
  const int64_t row = first + blockIdx.x;
  const T* const x = a.x + row * a.ldx;
  auto pieces = [&](auto&& f) {
    for (int64_t c = (int64_t)threadIdx.x * VEC; c < a.cols; c += 1024 * VEC) f(c);
  };
  float sum[1] = {0.0f};
  pieces([&](const int64_t c) {
    const auto v = row_piece<T>(x, c, a.cols);
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) s += (float)v[e];
    sum[0] += s;
  });
  norm_sums<1024, 1>(sum, part[0]);
  const float mean = sum[0] / a.count;
  float square[1] = {0.0f};
  pieces([&](const int64_t c) {
    const auto v = row_piece<T>(x, c, a.cols);
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float d = (float)v[e] - mean;
      if (c + e < a.cols) s += d * d;
    }
    square[0] += s;
  });
  norm_sums<1024, 1>(square, part[1]);
  const float rstd = 1.0f / sqrtf(square[0] / a.count + a.eps);
  if (threadIdx.x == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
  pieces([&](const int64_t c) {
    const auto v = row_piece<T>(x, c, a.cols);
    typename Core<T>::piece_t w, b;
    float out[VEC];
    if (a.w) w = row_piece<T>(a.w, c, a.cols);
    if (a.b) b = row_piece<T>(a.b, c, a.cols);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      float u = ((float)v[e] - mean) * rstd;
      if (a.w) u *= (float)w[e];
      if (a.b) u += (float)b[e];
      out[e] = u;
    }
    row_store<T, T>(a.y + row * a.ldy, c, a.cols, out);
  });
}

template <typename T>
struct NormBackward {
  const T *dy, *x, *w;                 // w null: 1
  int64_t lddy, ldx;
  const float *mean, *rstd;
  T* dx;                               // null: not wanted
  int64_t lddx;
  float* sums;                         // strips x 2 x cols: of dy h, of dy; null: not wanted
  int64_t rows, cols;
  float count;
};

// Rows strip, strip + strips, ... by a workgroup, each by LANES lanes; the sums over its rows stay in registers, and the next row is on its way
// while one is summed up.  Bytes bound it: 16384 x 4096 bf16 94 us (4.3 TB/s; without the next row on its way and with two pieces in 256 lanes 98);
// few rows, the barriers of one behind the other (777 x 1301 fp32 11 us).  Behind a row's end dy counts
// as zero, and with it everything that is summed: x as an element of the row, since from a zero there mean rstd could overflow.
template <typename T, int THREADS, int LANES, int P>
__global__ __launch_bounds__(THREADS) void norm_backward_kernel(const NormBackward<T> a) {
  typedef typename Core<T>::piece_t piece_t;
  constexpr int VEC = Core<T>::VEC, GROUPS = THREADS / LANES;
  constexpr bool AHEAD = THREADS * P < 2048;                   // as long as there are registers
  __shared__ float part[2][THREADS / 64][2];
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
  const int64_t step = (int64_t)gridDim.x * GROUPS;
  float dw[P][VEC] = {}, db[P][VEC] = {};
  piece_t d1[P], h1[P];
  float mean1 = 0.0f, rstd1 = 0.0f;
  auto get = [&](const int64_t row) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
      d1[p] = row_piece<T>(a.dy + row * a.lddy, (p * LANES + lane) * VEC, a.cols);
      h1[p] = row_piece_filled<T>(a.x + row * a.ldx, (p * LANES + lane) * VEC, a.cols);
    }
    mean1 = a.mean[row];
    rstd1 = a.rstd[row];
  };
  int turn = 0;
  int64_t row = (int64_t)blockIdx.x * GROUPS + group;          // the lanes of one row agree
  if (AHEAD && row < a.rows) get(row);
  for (; row < a.rows; row += step, turn ^= 1) {
    if (!AHEAD) get(row);
    piece_t d[P], h[P];
#pragma unroll
    for (int p = 0; p < P; ++p) d[p] = d1[p], h[p] = h1[p];
    const float mean = mean1, rstd = rstd1;
    if (AHEAD && row + step < a.rows) get(row + step);
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int p = 0; p < P; ++p) {
      piece_t w;
      if (a.w) w = row_piece<T>(a.w, (p * LANES + lane) * VEC, a.cols);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float g = (float)d[p][e], n = ((float)h[p][e] - mean) * rstd, u = a.w ? g * (float)w[e] : g;
        sum[0] += u;
        sum[1] += u * n;
        dw[p][e] += g * n;
        db[p][e] += g;
      }
    }
    if (!a.dx) continue;
    norm_sums<LANES, 2>(sum, part[turn]);
    const float m0 = sum[0] / a.count, m1 = sum[1] / a.count;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int64_t c = (p * LANES + lane) * VEC;
      if (c >= a.cols) break;
      piece_t w;
      float out[VEC];
      if (a.w) w = row_piece<T>(a.w, c, a.cols);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float g = (float)d[p][e], n = ((float)h[p][e] - mean) * rstd, u = a.w ? g * (float)w[e] : g;
        out[e] = rstd * (u - m0 - n * m1);
      }
      row_store<T, T>(a.dx + row * a.lddx, c, a.cols, out);
    }
  }
  if (!a.sums) return;
  float* const to = a.sums + (int64_t)blockIdx.x * 2 * a.cols;
  if constexpr (GROUPS == 1) {
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const int64_t c = (int64_t)(p * LANES + lane) * VEC + e;
        if (c < a.cols) to[c] = dw[p][e], to[a.cols + c] = db[p][e];
      }
  } else {
    // the groups' sums, added in their order, one of the two after the other
    __shared__ float all[GROUPS][P * LANES * VEC];
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      __syncthreads();
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int e = 0; e < VEC; ++e) all[group][(p * LANES + lane) * VEC + e] = which ? db[p][e] : dw[p][e];
      __syncthreads();
      for (int c = threadIdx.x; c < a.cols; c += THREADS) {
        float s = all[0][c];
#pragma unroll
        for (int g = 1; g < GROUPS; ++g) s += all[g][c];
        to[which * a.cols + c] = s;
      }
    }
  }
}

// Rows that no workgroup has registers for (the gradient of more than 8192 columns): dx, reading the row twice, for the most part from behind the L2
// caches both times (4096 x 16384 bf16: 95 us, 477 MB read where x and dy are 268) ...
template <typename T>
__global__ __launch_bounds__(1024) void norm_backward_long_kernel(const NormBackward<T> a, const int64_t first) {
  constexpr int VEC = Core<T>::VEC;
  __shared__ float part[16][2];
  const int64_t row = first + blockIdx.x;
  const T* const dy = a.dy + row * a.lddy;
  const T* const x = a.x + row * a.ldx;
  const float mean = a.mean[row], rstd = a.rstd[row];
  float sum[2] = {0.0f, 0.0f};
  for (int64_t c = (int64_t)threadIdx.x * VEC; c < a.cols; c += 1024 * VEC) {
    const auto d = row_piece<T>(dy, c, a.cols), h = row_piece_filled<T>(x, c, a.cols);
    typename Core<T>::piece_t w;
    if (a.w) w = row_piece<T>(a.w, c, a.cols);
    float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float u = a.w ? (float)d[e] * (float)w[e] : (float)d[e];
      s0 += u;
      s1 += u * (((float)h[e] - mean) * rstd);
    }
    sum[0] += s0;
    sum[1] += s1;
  }
  norm_sums<1024, 2>(sum, part);
  const float m0 = sum[0] / a.count, m1 = sum[1] / a.count;
  for (int64_t c = (int64_t)threadIdx.x * VEC; c < a.cols; c += 1024 * VEC) {
    const auto d = row_piece<T>(dy, c, a.cols), h = row_piece<T>(x, c, a.cols);
    typename Core<T>::piece_t w;
    float out[VEC];
    if (a.w) w = row_piece<T>(a.w, c, a.cols);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float u = a.w ? (float)d[e] * (float)w[e] : (float)d[e];
      out[e] = rstd * (u - m0 - ((float)h[e] - mean) * rstd * m1);
    }
    row_store<T, T>(a.dx + row * a.lddx, c, a.cols, out);
  }
}

// ... and the sums over each strip's rows, a piece of columns a thread, which read x and dy once more (the same: 62 us with the join).
template <typename T>
__global__ __launch_bounds__(NORM_THREADS) void norm_columns_kernel(const NormBackward<T> a, const int64_t strips) {
  constexpr int VEC = Core<T>::VEC;
  const int64_t across = (a.cols + VEC * NORM_THREADS - 1) / (VEC * NORM_THREADS), strip = blockIdx.x / across;
  const int64_t c = (blockIdx.x % across * NORM_THREADS + threadIdx.x) * VEC;
  if (c >= a.cols) return;
  float dw[VEC] = {}, db[VEC] = {};
  for (int64_t row = strip; row < a.rows; row += strips) {
    const auto d = row_piece<T>(a.dy + row * a.lddy, c, a.cols), x = row_piece<T>(a.x + row * a.ldx, c, a.cols);
    const float mean = a.mean[row], rstd = a.rstd[row];
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float g = (float)d[e];
      dw[e] += g * (((float)x[e] - mean) * rstd);
      db[e] += g;
    }
  }
  float* const to = a.sums + strip * 2 * a.cols;
#pragma unroll
  for (int e = 0; e < VEC; ++e)
    if (c + e < a.cols) to[c + e] = dw[e], to[a.cols + c + e] = db[e];
}

// dw and db: the strips' sums, added in one order, 64 threads a column, each with eight of its loads on their way at once: 512 strips of 4096
// columns 7 us (1024 strips, sixteen threads a column and one load after the other: 19).
constexpr int NORM_COLS = 16, NORM_JOIN = 64;

template <typename O>
__global__ __launch_bounds__(NORM_COLS * NORM_JOIN) void norm_join_kernel(const float* __restrict__ sums, const int64_t strips, const int64_t cols,
                                                                          O* __restrict__ dw, O* __restrict__ db, const int64_t first) {
  __shared__ float part[2][NORM_JOIN][NORM_COLS];
  const int t = threadIdx.x / NORM_COLS, c = threadIdx.x % NORM_COLS;
  const int64_t col = (first + blockIdx.x) * NORM_COLS + c;
  float sw = 0.0f, sb = 0.0f;
  if (col < cols) {
    const float* from = sums + t * 2 * cols + col;
    int64_t s = t;
    for (; s + 3 * NORM_JOIN < strips; s += 4 * NORM_JOIN) {
      float w[4], b[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        w[u] = from[u * (2 * NORM_JOIN * cols)];
        b[u] = from[u * (2 * NORM_JOIN * cols) + cols];
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) sw += w[u], sb += b[u];
      from += 4 * (2 * NORM_JOIN * cols);
    }
    for (; s < strips; s += NORM_JOIN, from += 2 * NORM_JOIN * cols) sw += from[0], sb += from[cols];
  }
  part[0][t][c] = sw;
  part[1][t][c] = sb;
  __syncthreads();
  if (t < 2 && col < cols) {
    O* const to = t ? db : dw;
    float v = part[t][0][c];
#pragma unroll
    for (int r = 1; r < NORM_JOIN; ++r) v += part[t][r][c];
    if (to) to[col] = (O)v;
  }
}

}  // namespace mdet
