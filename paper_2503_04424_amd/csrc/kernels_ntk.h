// Gram matrix K = J J^T of a network's Jacobian (the NTK, Sec. 2.1), without J.
//
// A dense layer z = W a + b contributes to the derivative of output r at sample i the outer product of g = df_r / dz with
// a, and g itself for b.  The inner product of two such is (a . a' + 1) (g . g'), so with the layers' inputs a_l (n x p_l)
// and gradients g_l (n d x q_l, row i d + r: sample i, output r)
//
//   K[(i, r), (j, s)] = scale sum_l (a_l,i . a_l,j + bias) (g_l,ir . g_l,js)
//
// J would have sum_l (p_l + 1) q_l columns; here a layer takes n^2 p_l + (n d)^2 q_l operations for the lower triangle,
// which is all that the log-determinant reads and all that is written.  The arithmetic is K's type: fp32 (operands in 16
// or 32 bits) or fp64.
#pragma once
#include "kernels_gemm.h"

namespace mdet {

constexpr int NTK_LAYERS = 32;         // a launch's, so that they fit the kernel's arguments

template <typename T>
struct NtkLayers {
  int count;
  int64_t p[NTK_LAYERS], q[NTK_LAYERS];
  const T* a[NTK_LAYERS];
  const T* g[NTK_LAYERS];
  int64_t lda[NTK_LAYERS], ldg[NTK_LAYERS];
};

// Element i of a matrix in type S, as a double; the conversions to fp64 are exact.
template <typename S>
__global__ __launch_bounds__(256) void ntk_widen_kernel(const S* __restrict__ from, const int64_t ld, double* __restrict__ to, const int64_t rows,
                                                        const int64_t cols, const int64_t ldto) {
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t i = id / ldto, k = id % ldto;
  if (i < rows) to[i * ldto + k] = k < cols ? (double)from[i * ld + k] : 0.0;
}

// Block number t of the lower triangle, row by row.
__device__ __forceinline__ void ntk_block(const int64_t t, int64_t& bi, int64_t& bj) {
  bi = (int64_t)((sqrt(8.0 * (double)t + 1.0) - 1.0) * 0.5);
  while (bi * (bi + 1) / 2 > t) --bi;
  while ((bi + 1) * (bi + 2) / 2 <= t) ++bi;
  bj = t - bi * (bi + 1) / 2;
}

// One 64 x 64 block: total += (a a^T + bias) * (g g^T), layer after layer, written once.  Rows of a: that of sample i
// stands for rows i d .. i d + d - 1 of K.
template <typename T>
struct NtkRows {                       // rows i / d of a, as an operand whose rows repeat
  const T* p;
  int64_t stride, rows, d;
};

template <typename T>
__device__ __forceinline__ void ntk_stage(typename Core<T>::piece_t (&to)[PLAIN_TILE][GEMM_PIECES + 1], const NtkRows<T>& o, const int64_t i0,
                                          const int64_t k0, const int64_t kend) {
  constexpr int VEC = Core<T>::VEC;
#pragma unroll
  for (int s = 0; s < PLAIN_TILE * GEMM_PIECES / PLAIN_THREADS; ++s) {
    const int id = s * PLAIN_THREADS + (int)threadIdx.x, row = id / GEMM_PIECES, piece = id % GEMM_PIECES;
    const int64_t i = i0 + row, k = k0 + piece * VEC;
    typename Core<T>::piece_t v;
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = i < o.rows && k + e < kend ? o.p[i / o.d * o.stride + k + e] : T(0);
    to[row][piece] = v;
  }
}

template <typename T>
__device__ __forceinline__ void ntk_accumulate(typename Core<T>::acc_t (&acc)[2][2], PlainLds<T>& lds, const NtkRows<T>& o, const int64_t row0,
                                               const int64_t col0, const int64_t kend) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int rw = (wave >> 1) * 32 + (lane & 15), cw = (wave & 1) * 32 + (lane & 15);
  for (int64_t k = 0; k < kend; k += GEMM_PIECES * Core<T>::VEC) {
    __syncthreads();
    ntk_stage<T>(lds.r, o, row0, k, kend);
    ntk_stage<T>(lds.c, o, col0, k, kend);
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int piece = 4 * h + (lane >> 4);
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int b = 0; b < 2; ++b) Core<T>::mma(lds.c[cw + 16 * a][piece], lds.r[rw + 16 * b][piece], acc[a][b]);
    }
  }
}

template <typename T>
__global__ __launch_bounds__(PLAIN_THREADS) void ntk_plain_kernel(const NtkLayers<T> layers, const int64_t n, const int64_t d,
                                                                  const typename Core<T>::acc1_t bias, const typename Core<T>::acc1_t scale,
                                                                  const int accumulate, typename Core<T>::acc1_t* __restrict__ K, const int64_t ldk) {
  typedef typename Core<T>::acc_t acc_t;
  __shared__ PlainLds<T> lds;
  int64_t bi, bj;
  ntk_block(blockIdx.x, bi, bj);
  const int64_t row0 = bi * PLAIN_TILE, col0 = bj * PLAIN_TILE, N = n * d;
  acc_t total[2][2] = {};
  for (int l = 0; l < layers.count; ++l) {
    acc_t first[2][2] = {}, second[2][2] = {};
    ntk_accumulate<T>(first, lds, NtkRows<T>{layers.a[l], layers.lda[l], N, d}, row0, col0, layers.p[l]);
    ntk_accumulate<T>(second, lds, NtkRows<T>{layers.g[l], layers.ldg[l], N, 1}, row0, col0, layers.q[l]);
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int b = 0; b < 2; ++b) total[a][b] += (first[a][b] + bias) * second[a][b];
  }
  plain_each<T>([&](int a, int b, int e, int i, int j) {
    const int64_t I = row0 + i, J = col0 + j;
    if (I >= N || J > I) return;
    auto v = total[a][b][e] * scale;
    if (accumulate) v += K[I * ldk + J];
    K[I * ldk + J] = v;
  });
}

}  // namespace mdet
