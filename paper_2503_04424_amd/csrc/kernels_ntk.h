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
  uint32_t near_a, near_g, straight_a, straight_g;   // bit l: see Operand
};
static_assert(NTK_LAYERS <= 32, "a bit for each");

// Element i of a matrix in type S, as a double; the conversions to fp64 are exact.
template <typename S>
__global__ __launch_bounds__(256) void ntk_widen_kernel(const S* __restrict__ from, const int64_t ld, double* __restrict__ to, const int64_t rows,
                                                        const int64_t cols, const int64_t ldto, const int64_t first) {
  const int64_t id = (first + blockIdx.x) * 256 + threadIdx.x;
  const int64_t i = id / ldto, k = id % ldto;
  if (i < rows) to[i * ldto + k] = k < cols ? (double)from[i * ld + k] : 0.0;
}

// Blocks of the lower triangle of `rows` rows of blocks, and where number t of them is: bands of eight rows of blocks, each
// column by column and the triangle at its end row by row, so that neighbours read the same operands.
__host__ __device__ __forceinline__ int64_t ntk_blocks(const int64_t rows) { return rows * (rows + 1) / 2; }
__device__ __forceinline__ void ntk_block(const int64_t t, const int64_t rows, int64_t& bi, int64_t& bj) {
  // 32 r^2 + 4 r blocks stand before band r
  int64_t r = (int64_t)((sqrt(16.0 + 128.0 * (double)t) - 4.0) * (1.0 / 64.0));
  while (32 * r * r + 4 * r > t) --r;
  while (32 * (r + 1) * (r + 1) + 4 * (r + 1) <= t) ++r;
  const int64_t u = t - (32 * r * r + 4 * r);
  const int height = rows - 8 * r < 8 ? (int)(rows - 8 * r) : 8;
  if (u < height * 8 * r) {
    bi = 8 * r + u % height;
    bj = u / height;
  } else {
    const int v = (int)(u - height * 8 * r);
    int i = 0;
    while ((i + 1) * (i + 2) / 2 <= v) ++i;
    bi = 8 * r + i;
    bj = 8 * r + v - i * (i + 1) / 2;
  }
}

// first[l] = a_l a_l^T + bias, lower triangle of n x n, for networks of several outputs: every pair of samples' product
// serves outputs^2 elements of K.
template <typename T, typename S, bool DIRECT>
__global__ __launch_bounds__(S::THREADS) void ntk_first_kernel(const NtkLayers<T> layers, const int64_t n, const typename Core<T>::acc1_t bias,
                                                               typename Core<T>::acc1_t* __restrict__ first) {
  __shared__ __attribute__((aligned(16))) char lds[S::NB * S::SLAB];
  const int64_t rows = (n + S::BM - 1) / S::BM, blocks = ntk_blocks(rows);
  const int64_t t = gemm_tile_number(blockIdx.x, blocks * layers.count);
  if (t < 0) return;
  int64_t bi, bj;
  ntk_block(t % blocks, rows, bi, bj);
  const int l = (int)(t / blocks);
  const Operand<T> a{layers.a[l], layers.lda[l], n, (layers.near_a >> l & 1) != 0, (layers.straight_a >> l & 1) != 0};
  typename Core<T>::acc_t acc[S::TN][S::TM] = {};
  TileStream<T, S, false, false, DIRECT> stream(lds);
  auto none = [] { return false; };
  stream.set(a, a, bi * S::BM, bj * S::BN, 0, layers.p[l]);
  stream.begin(none);
  stream.run(acc, stream.slabs(0, layers.p[l]), none);
  typename Core<T>::acc1_t* const to = first + l * n * n;
  tile_each<T, S>([&](int a0, int b0, int e, int i, int j) {
    const int64_t I = bi * S::BM + i, J = bj * S::BN + j;
    if (I < n && J <= I) to[I * n + J] = acc[a0][b0][e] + bias;
  });
}

// Blocks `begin` .. `begin` + `count` - 1 of K.  With PARTS the launch's workgroups take the four quarters (64 x 64) of blocks of
// twice the tile's size.  FIRST: the first factors stand in `first`; otherwise (one output) both products are formed here, one
// after the other, and multiplied in registers.  The sum over layers stays in registers, K is written once.
// The matrix cores bound large orders of one output (n = 8192, three layers: fp64 2.87 ms, 66 TFLOP/s; fp32 1.47 ms, 129),
// the chain of short products small ones (n = 512: 18 us) and those of several outputs (1000 x 10 bf16, four layers: 376 us).
template <typename T, typename S, bool DIRECT, bool FIRST, bool PARTS>
__global__ __launch_bounds__(S::THREADS) void ntk_gram_kernel(const NtkLayers<T> layers, const int64_t begin, const int64_t count, const int64_t n, const int d,
                                                              const typename Core<T>::acc1_t bias, const typename Core<T>::acc1_t scale,
                                                              const int accumulate, const typename Core<T>::acc1_t* __restrict__ first,
                                                              typename Core<T>::acc1_t* __restrict__ K, const int64_t ldk) {
  typedef typename Core<T>::acc_t acc_t;
  __shared__ __attribute__((aligned(16))) char lds[S::NB * S::SLAB];
  constexpr int EACH = PARTS ? 4 : 1, EDGE = PARTS ? 2 : 1;
  const int64_t N = n * d, rows = (N + EDGE * S::BM - 1) / (EDGE * S::BM);
  const int64_t t = gemm_tile_number(blockIdx.x, EACH * count);
  if (t < 0) return;
  int64_t bi, bj;
  ntk_block(begin + t / EACH, rows, bi, bj);
  if constexpr (PARTS) {
    bi = 2 * bi + (t >> 1 & 1);
    bj = 2 * bj + (t & 1);
    if (bj > bi) return;
  }
  const int64_t row0 = bi * S::BM, col0 = bj * S::BN;
  if (row0 >= N || col0 >= N) return;              // a block may reach over the matrix's edge
  acc_t total[S::TN][S::TM] = {};
  // The first factors of a block's samples go through LDS: every one serves d^2 elements.  A large block's are those of three
  // outputs or more, so that two workgroups' LDS fits a compute unit.
  constexpr int SAMPLES = !FIRST ? 1 : S::BM == 128 ? 44 : S::BM / 2 + 1, EACH_THREAD = (SAMPLES * SAMPLES + S::THREADS - 1) / S::THREADS;
  __shared__ typename Core<T>::acc1_t patch[SAMPLES * SAMPLES];
  int patch_row[S::TM], patch_col[S::TN][4], down = 0, across = 0;
  int64_t sample0 = 0;                             // of the patch's first element in `first`
  if constexpr (FIRST) {
    auto of = [&](const int64_t i) { return (int)((uint32_t)(i < N ? i : N - 1) / (uint32_t)d); };
    const int i0 = of(row0), j0 = of(col0);
    down = of(row0 + S::BM - 1) - i0 + 1;
    across = of(col0 + S::BN - 1) - j0 + 1;
    sample0 = i0 * n + j0;
    tile_each<T, S>([&](int a, int b, int e, int i, int j) {
      if (a == 0 && e == 0) patch_row[b] = (of(row0 + i) - i0) * across;
      if (b == 0) patch_col[a][e] = of(col0 + j) - j0;
    });
  }
  auto of_a = [&](const int l) { return Operand<T>{layers.a[l], layers.lda[l], N, (layers.near_a >> l & 1) != 0, (layers.straight_a >> l & 1) != 0}; };
  auto of_g = [&](const int l) { return Operand<T>{layers.g[l], layers.ldg[l], N, (layers.near_g >> l & 1) != 0, (layers.straight_g >> l & 1) != 0}; };
  TileStream<T, S, false, false, DIRECT> stream(lds);
  // the products in their order: g_l g_l^T, then (one output) a_l a_l^T
  int product = 0;
  auto next = [&] {
    const int l = FIRST ? product : product >> 1;
    if (l >= layers.count) return false;
    const bool second = FIRST || !(product & 1);
    const Operand<T> o = second ? of_g(l) : of_a(l);
    stream.set(o, o, row0, col0, 0, second ? layers.q[l] : layers.p[l]);
    ++product;
    return true;
  };
  stream.begin(next);
  for (int l = 0; l < layers.count; ++l) {
    acc_t second[S::TN][S::TM] = {};
    // brought beside the products where there are registers for it
    constexpr bool EARLY = FIRST && sizeof(T) < 8;
    typename Core<T>::acc1_t part[EACH_THREAD];
    auto bring_part = [&] {
#pragma unroll
      for (int v = 0; v < EACH_THREAD; ++v) {
        const int at = v * S::THREADS + (int)threadIdx.x;
        // above the diagonal there are none; nothing is stored there
        part[v] = at < down * across ? first[(l * n + at / across) * n + sample0 + at % across] : 0;
      }
    };
    if constexpr (EARLY) bring_part();
    stream.run(second, stream.slabs(0, layers.q[l]), next);
    if constexpr (FIRST) {
      if constexpr (!EARLY) bring_part();
      __syncthreads();                             // the layer before has been read
#pragma unroll
      for (int v = 0; v < EACH_THREAD; ++v) {
        const int at = v * S::THREADS + (int)threadIdx.x;
        if (at < down * across) patch[at] = part[v];
      }
      __syncthreads();
#pragma unroll
      for (int b = 0; b < S::TM; ++b)
#pragma unroll
        for (int a = 0; a < S::TN; ++a)
#pragma unroll
          for (int e = 0; e < 4; ++e) total[a][b][e] += patch[patch_row[b] + patch_col[a][e]] * second[a][b][e];
    } else {
      acc_t one[S::TN][S::TM] = {};
      stream.run(one, stream.slabs(0, layers.p[l]), next);
#pragma unroll
      for (int a = 0; a < S::TN; ++a)
#pragma unroll
        for (int b = 0; b < S::TM; ++b) total[a][b] += (one[a][b] + bias) * second[a][b];
    }
  }
  // four neighbours of a row in one store where a lane has them
  typedef typename Core<T>::acc1_t four_t __attribute__((ext_vector_type(4)));
  const bool vec = sizeof(typename Core<T>::acc1_t) == 4 && (uintptr_t)K % 16 == 0 && ldk % 4 == 0;
#pragma unroll
  for (int b = 0; b < S::TM; ++b)
#pragma unroll
    for (int a = 0; a < S::TN; ++a) {
      const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
      const int64_t I = row0 + (wave / S::WN * S::TM + b) * 16 + (lane & 15), J = col0 + (wave % S::WN * S::TN + a) * 16;
      if (I >= N) continue;
      if (vec && J + Core<T>::col(lane, 3) <= I) {
        four_t* const to = reinterpret_cast<four_t*>(K + I * ldk + J + Core<T>::col(lane, 0));
        four_t v = total[a][b] * scale;
        if (accumulate) v += *to;
        *to = v;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int64_t j = J + Core<T>::col(lane, e);
          if (j > I) continue;
          auto v = total[a][b][e] * scale;
          if (accumulate) v += K[I * ldk + j];
          K[I * ldk + j] = v;
        }
      }
    }
}

}  // namespace mdet
