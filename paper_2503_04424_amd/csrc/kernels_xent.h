// Softmax cross entropy of a linear layer over a large vocabulary, and its gradient, without its logits in memory.
//
//   z = x W^T + b;  lse_i = log(sum over j of exp(z_ij));  loss_i = lse_i - z_i,t_i
//   e_ij = g_i (exp(z_ij - lse_i) - [j = t_i]);  dx = e W;  dW = e^T x;  db = column sums of e
//
// The target's e is -g (1 - exp(-loss)), from the loss itself: the loss is formed from the difference of two logits, while lse is rounded to its
// own size, and of a row that is sure of its target no more than that rounding would be left of exp(z_t - lse) - 1 (126 words, the target 14 above
// the others: 0.9 % off at logits of 60, 17 % at 1000).
//
// Forward, each tile of z stays in the accumulators: what leaves it are each row's largest logit M and the sum of exp(z - M) over the
// tile's columns (a strip), joined by a second launch, and the logit of the target.  Backward, z is formed once more in front
// of e, a piece of the vocabulary at a time; or, where the forward pass kept them, exp(z - M) is read back (M is the strip's: nothing
// overflows, and what is rounded keeps its relative precision), which spares that product.
//
// Sums and everything behind them are fp32; e is rounded to the operands' type in front of its two products, db sums the unrounded one.  Where dW
// is wanted in 32 bits of operands in 16, that rounding would be all of its error: e goes in as two (fp16) or three (bf16) numbers that add up
// to it, their rows one behind the other beside as many copies of x, a sum over two or three times the rows.
// In 16 bits e is divided by the largest |g|, and the products multiplied by it: of a mean, whose g are all alike, the same rounding of 1 / count
// would be in every row otherwise (a row that is not sure of its target has e = -g there, which is nearly all of its dx; the error of dx and dW
// for 2048 rows of 512 over 16384 words in bf16 0.0025 and 0.0020 of their norm, of which 0.0017 are the results' own rounding).  In fp16 by
// 2^-14 of it: e would vanish below 2^-24, where most probabilities of a large vocabulary lie.
//
// Rows whose target lies outside of the vocabulary, or is `ignore`, do not count: loss 0, e exactly 0 whatever their logits are, and zeros
// in the place of their x in dW, so that nothing of them comes through.
#pragma once
#include "kernels_gemm.h"
#include "kernels_rows.h"

namespace mdet {

struct XentTargets {
  const void* target;
  int bits;                            // 32 or 64
  int64_t ignore, vocab;
};
// The target of row i, in two steps, so that the loads of several rows can be on their way beside a product: what is in memory, then what it
// says; -1 if the row does not count.
__device__ __forceinline__ int64_t xent_raw(const XentTargets& t, const int64_t i) {
  const int32_t* const p = static_cast<const int32_t*>(t.target) + (t.bits == 32 ? i : 2 * i);
  const uint32_t low = (uint32_t)p[0], high = (uint32_t)p[t.bits == 32 ? 0 : 1];
  return (int64_t)((uint64_t)high << 32 | low);
}
__device__ __forceinline__ int64_t xent_said(const XentTargets& t, const int64_t raw) {
  const int64_t v = t.bits == 32 ? (int64_t)(int32_t)raw : raw;
  return v < 0 || v >= t.vocab || v == t.ignore ? -1 : v;
}

__device__ __forceinline__ int64_t xent_target(const XentTargets& t, const int64_t i) { return xent_said(t, xent_raw(t, i)); }

// exp(z - top) is __expf(z - xent_from(top)), from the difference: 2^-23 of its size is what the result is off by, however large both are (the
// product of each with log2(e) apart, one multiplication and addition, would round to more than 2^128 from logits of 1e10 on).  Zero for
// z = -inf, also where top is the largest of some z that are all -inf.
__device__ __forceinline__ float xent_from(const float top) { return top == -INFINITY ? 0.0f : top; }
__device__ __forceinline__ float xent_exp(const float z, const float top) { return __expf(z - xent_from(top)); }

// What is kept of exp(z - top): numbers up to 1, to 11 bits for operands in bf16 (fewer would add to what rounding e costs), to 24 otherwise.
template <typename T> struct XentKept { typedef float type; };
template <> struct XentKept<__bf16> { typedef _Float16 type; };

struct XentStrip {                     // of a row: its largest logit among a strip's columns, and the sum of exp(z - top)
  float top, sum;
};

template <typename T>
struct XentForward {
  XentTargets t;
  const T* bias;                       // null: none
  XentStrip* strips;                   // rows x across
  int64_t across;
  float* picked;                       // of the rows that count: the target's logit; behind the join their loss, for the gradient
  typename XentKept<T>::type* exps;    // rows x ldexps, exp(z - top); null: not kept
  int64_t ldexps, rows, cols;
};

// The units of a launch (tiles, or parts of a sum over k of one), which its workgroups take one after the other, gridDim.x apart, so that one
// launch fills the device once: the first `whole` are tiles, which go round the chiplets as gemm_tile_number says, each of the others is one
// of `splits` parts of a tile, kpart of k long.  Fewer than 2^31 of all.
struct XentUnits {
  int down, across, whole, units;      // units: whole + splits (tiles - whole)
  int splits;
  int64_t k, kpart;
  float* parts;                        // of the units behind the whole ones: BM x BN each
};
struct XentUnit {
  int bi, bj, part;                    // part: -1, the tile is whole
  int64_t k0, kend;
};
// Unit number `id` of a launch, which may name none.
__device__ __forceinline__ void xent_place(const XentUnits& u, const int t, int& bi, int& bj) {
  // as gemm_tile_place
  const int group = t / (8 * u.across), in = t - group * 8 * u.across, left = u.down - 8 * group, rows = left < 8 ? left : 8;
  bj = in / rows;
  bi = 8 * group + in - bj * rows;
}
__device__ __forceinline__ bool xent_unit(const XentUnits& u, int& id, XentUnit& x) {
  const int per = (u.whole + 7) / 8, round = 8 * per;
  int t = -1;
  for (; id < round; id += gridDim.x) {
    t = (id & 7) * per + (id >> 3);
    if (t < u.whole) break;
    t = -1;
  }
  x.k0 = 0;
  x.kend = u.k;
  x.part = -1;
  if (t < 0) {
    x.part = id - round;
    if (x.part >= u.units - u.whole) return false;
    t = u.whole + x.part / u.splits;
    x.k0 = x.part % u.splits * u.kpart;
    x.kend = x.k0 + u.kpart < u.k ? x.k0 + u.kpart : u.k;
  }
  xent_place(u, t, x.bi, x.bj);
  return true;
}
// f(unit, run) for each of the workgroup's units, where run(acc) adds up its product.  The first slab of a unit is brought while the one before
// it is on its way out (at 256 x 256, 64 of k are 1.7 us of products; a tile by itself waited 9 us more at its ends).  Where operands go
// through registers none are left for that: a workgroup has one unit then.  early(unit): what may be on its way beside the product.
template <typename T, typename S, bool ROUTER, bool COUTER, bool DIRECT, typename E, typename F>
__device__ __forceinline__ void xent_units(char* const lds, const Operand<T>& r, const Operand<T>& c, const XentUnits& u, E&& early, F&& f) {
  TileStream<T, S, ROUTER, COUTER, DIRECT> stream(lds);
  int id = blockIdx.x;
  XentUnit now, then;
  bool more = xent_unit(u, id, then), fresh = more;
  auto next = [&] {
    if (!fresh) return false;
    fresh = false;
    stream.set(r, c, (int64_t)then.bi * S::BM, (int64_t)then.bj * S::BN, then.k0, then.kend);
    return true;
  };
  stream.begin(next);
  while (more) {
    now = then;
    more = false;
    if constexpr (DIRECT) {
      id += gridDim.x;
      more = fresh = xent_unit(u, id, then);
    }
    early(now);
    typename Core<T>::acc_t acc[S::TN][S::TM] = {};
    if constexpr (sizeof(T) == 4) {
      // in 32 bits the sums' own rounding counts: 1024 terms at a time, which are then added up
      for (int left = stream.slabs(now.k0, now.kend); left > 0; left -= 32) {
        typename Core<T>::acc_t some[S::TN][S::TM] = {};
        const int count = left < 32 ? left : 32;
        stream.run(some, count, next);
#pragma unroll
        for (int a = 0; a < S::TN; ++a)
#pragma unroll
          for (int b = 0; b < S::TM; ++b) acc[a][b] += some[a][b];
      }
    } else if constexpr (DIRECT && S::BM == 256) stream.run_rolling(acc, stream.slabs(now.k0, now.kend), next);
    else stream.run(acc, stream.slabs(now.k0, now.kend), next);
    // of a sum over nothing no slab was brought, and nothing is on its way
    fresh = false;
    f(now, acc);
  }
}

// The largest, or the sum, of the four lanes 16 apart, in each of them.
template <typename F>
__device__ __forceinline__ float xent_across(const float v, F&& f) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  const float w = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(w), __float_as_uint(w), false, false);
  return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Four neighbours each of two blocks of 16 columns, in 16 bits: eight neighbours in their place, of the first block for lanes 0 .. 15 and 32 .. 47, of the
// second for the others.  A row's 64 bytes leave in one store; with eight bytes a lane the stores of a tile of 128 KB took 8 us.
template <typename O>
struct XentEight {
  typedef O four_t __attribute__((ext_vector_type(4)));
  typedef O eight_t __attribute__((ext_vector_type(8)));
  typedef unsigned two_t __attribute__((ext_vector_type(2)));
  typedef unsigned quad_t __attribute__((ext_vector_type(4)));
  // Column of a lane's eight, counted from the first block's.
  static __device__ __forceinline__ int col() {
    const int g = threadIdx.x >> 4 & 3;
    return 16 * (g & 1) + 8 * (g >> 1);
  }
  static __device__ __forceinline__ eight_t of(const four_t& a, const four_t& b) {
    const two_t x = __builtin_bit_cast(two_t, a), y = __builtin_bit_cast(two_t, b);
    const auto p = __builtin_amdgcn_permlane16_swap(x[0], y[0], false, false), q = __builtin_amdgcn_permlane16_swap(x[1], y[1], false, false);
    return __builtin_bit_cast(eight_t, quad_t{p[0], q[0], p[1], q[1]});
  }
};

// A row's block of S::TN * 16 columns from `col` on (a multiple of 16; `limit` columns in all, rows on 16 bytes and whole pieces of 8 long),
// value(a) the four of block a that this lane has.
template <typename T, int TN, typename F>
__device__ __forceinline__ void xent_store(T* const row, const int64_t col, const int64_t limit, const bool there, F&& value) {
  typedef T t4 __attribute__((ext_vector_type(4)));
  if constexpr (sizeof(T) == 2 && TN % 2 == 0) {
#pragma unroll
    for (int a = 0; a < TN; a += 2) {
      const auto v = XentEight<T>::of(value(a), value(a + 1));
      const int64_t j = col + 16 * a + XentEight<T>::col();
      if (there && j < limit) *reinterpret_cast<typename XentEight<T>::eight_t*>(row + j) = v;
    }
  } else {
#pragma unroll
    for (int a = 0; a < TN; ++a) {
      const int64_t j = col + 16 * a + 4 * (threadIdx.x >> 4 & 3);
      const t4 v = value(a);
      if (there && j < limit) *reinterpret_cast<t4*>(row + j) = v;
    }
  }
}

// Tiles of logits, and what is left of each of their rows: a strip for each of the wavefronts beside each other, so that no wavefront waits
// for another behind the product.  The matrix cores and the power they draw bound long rows (8192 x 4096 over 131072 words bf16 6.4 to 6.9 ms,
// 1.28 to 1.38 PFLOP/s; the library's product alone 5.98), the ends of a tile short ones (4096 x 1024 over 50003: 370 to 450 us, 0.93 to 1.13).
template <typename T, typename S, bool DIRECT>
__global__ __launch_bounds__(S::THREADS) void xent_forward_kernel(const Operand<T> r, const Operand<T> c, const XentForward<T> o, const XentUnits u) {
  typedef typename Core<T>::acc_t acc_t;
  typedef typename XentKept<T>::type K;
  typedef K k4 __attribute__((ext_vector_type(4)));
  constexpr int STRIP = S::TN * 16;
  __shared__ __attribute__((aligned(16))) char lds[S::NB * S::SLAB];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int wrow = wave / S::WN * (S::TM * 16) + (lane & 15), quad = 4 * (lane >> 4);
  int64_t raw[S::TM];                  // the rows' targets
  auto early = [&](const XentUnit& x) {
#pragma unroll
    for (int b = 0; b < S::TM; ++b) {
      const int64_t i = (int64_t)x.bi * S::BM + wrow + 16 * b;
      raw[b] = xent_raw(o.t, i < o.rows ? i : o.rows - 1);
    }
  };
  xent_units<T, S, false, false, DIRECT>(lds, r, c, u, early, [&](const XentUnit& x, acc_t (&acc)[S::TN][S::TM]) {
    const int64_t row0 = (int64_t)x.bi * S::BM + wrow, strip = (int64_t)x.bj * S::WN + wave % S::WN, col0 = strip * STRIP;
    int at[S::TM];                     // counted from this lane's first column on
#pragma unroll
    for (int b = 0; b < S::TM; ++b) {
      const int64_t t = xent_said(o.t, raw[b]) - (col0 + quad);
      at[b] = t >= 0 && t < STRIP && row0 + 16 * b < o.rows ? (int)t : -1;
    }
    if (o.bias || ((int64_t)x.bj + 1) * S::BN > o.cols) {
#pragma unroll
      for (int a = 0; a < S::TN; ++a)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int64_t j = col0 + quad + 16 * a + e;
          const bool there = j < o.cols;
          const float add = o.bias && there ? (float)o.bias[j] : 0.0f;
#pragma unroll
          for (int b = 0; b < S::TM; ++b) acc[a][b][e] = there ? acc[a][b][e] + add : -INFINITY;
        }
    }
#pragma unroll
    for (int b = 0; b < S::TM; ++b) {
      const int64_t i = row0 + 16 * b;
      if (__any(at[b] >= 0)) {
#pragma unroll
        for (int a = 0; a < S::TN; ++a)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (at[b] == 16 * a + e) o.picked[i] = acc[a][b][e];
      }
      float top = -INFINITY;
#pragma unroll
      for (int a = 0; a < S::TN; ++a)
#pragma unroll
        for (int e = 0; e < 4; ++e) top = fmaxf(top, acc[a][b][e]);
      top = xent_across(top, [](const float p, const float q) { return fmaxf(p, q); });
      const float from = xent_from(top);
      float sum = 0.0f;
#pragma unroll
      for (int a = 0; a < S::TN; ++a)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          acc[a][b][e] = __expf(acc[a][b][e] - from);
          sum += acc[a][b][e];
        }
      sum = xent_across(sum, [](const float p, const float q) { return p + q; });
      if (lane < 16 && i < o.rows && strip < o.across) o.strips[i * o.across + strip] = XentStrip{top, sum};
      // rows are ceil(cols / 8) 8 long or more: what is written behind their end is zero
      if (o.exps)
        xent_store<K, S::TN>(o.exps + i * o.ldexps, col0, o.cols, i < o.rows, [&](const int a) {
          return k4{(K)acc[a][b][0], (K)acc[a][b][1], (K)acc[a][b][2], (K)acc[a][b][3]};
        });
    }
  });
}

// Up to 16 rows: W is read once, GROUPS times 16 rows of it by a workgroup whose wavefronts share k; a piece of x serves all of the groups.  A
// strip is 16 columns, of a wavefront.  Bytes of W bound it: one row over 131072 words of 4096 in bf16 180 us (6 TB/s), 5 rows over 50003 of 1024 23.
constexpr int XENT_WAVES = 4;

template <typename T, int GROUPS>
__global__ __launch_bounds__(64 * XENT_WAVES) void xent_forward_rows_kernel(const Operand<T> x, const Operand<T> w, const int64_t k, const XentForward<T> o) {
  constexpr int WAVES = XENT_WAVES;
  typedef typename Core<T>::piece_t piece_t;
  typedef typename Core<T>::acc_t acc_t;
  constexpr int VEC = Core<T>::VEC, STEP = 4 * VEC, UNROLL = GROUPS == 4 ? 4 : 8;
  __shared__ acc_t part[WAVES][GROUPS][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), i = lane & 15, g = lane >> 4;
  // rows behind the last are not stored
  const T* wp[GROUPS];
#pragma unroll
  for (int q = 0; q < GROUPS; ++q) {
    const int64_t j = ((int64_t)blockIdx.x * GROUPS + q) * 16 + i;
    wp[q] = w.p + (j < w.rows ? j : w.rows - 1) * w.stride + g * VEC;
  }
  const T* const xp = x.p + (i < x.rows ? i : x.rows - 1) * x.stride + g * VEC;
  acc_t acc[GROUPS] = {};
  const int64_t steps = k / STEP, each = (steps + WAVES - 1) / WAVES;
  int64_t s = wave * each;
  const int64_t end = s + each < steps ? s + each : steps;
  auto some = [&](auto count) {
    constexpr int U = decltype(count)::value;
    piece_t wf[U][GROUPS], xf[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int q = 0; q < GROUPS; ++q) __builtin_memcpy(&wf[u][q], wp[q] + (s + u) * STEP, 16);
      __builtin_memcpy(&xf[u], xp + (s + u) * STEP, 16);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int q = 0; q < GROUPS; ++q) Core<T>::mma(wf[u][q], xf[u], acc[q]);
  };
  for (; s + UNROLL <= end; s += UNROLL) some(std::integral_constant<int, UNROLL>{});
  for (; s < end; ++s) some(std::integral_constant<int, 1>{});
  if (wave == WAVES - 1 && steps * STEP < k) {                 // what is left over, element by element
    const int64_t from = steps * STEP;
    piece_t wf[GROUPS] = {}, xf = {};
#pragma unroll
    for (int e = 0; e < VEC; ++e)
      if (from + g * VEC + e < k) {
        xf[e] = xp[from + e];
#pragma unroll
        for (int q = 0; q < GROUPS; ++q) wf[q][e] = wp[q][from + e];
      }
#pragma unroll
    for (int q = 0; q < GROUPS; ++q) Core<T>::mma(wf[q], xf, acc[q]);
  }
#pragma unroll
  for (int q = 0; q < GROUPS; ++q) part[wave][q][lane] = acc[q];
  __syncthreads();
  if (wave >= GROUPS) return;
  acc_t sum = part[0][wave][lane];
#pragma unroll
  for (int p = 1; p < WAVES; ++p) sum += part[p][wave][lane];
  const int64_t strip = (int64_t)blockIdx.x * GROUPS + wave, c = strip * 16 + 4 * g;
  const int64_t target = i < o.rows ? xent_target(o.t, i) : -1;
  float z[4], top = -INFINITY, total = 0.0f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    z[e] = c + e < o.cols ? sum[e] + (o.bias ? (float)o.bias[c + e] : 0.0f) : -INFINITY;
    top = fmaxf(top, z[e]);
    if (c + e == target) o.picked[i] = z[e];
  }
  top = fmaxf(top, __shfl_xor(top, 16, 64));
  top = fmaxf(top, __shfl_xor(top, 32, 64));
  const float from = xent_from(top);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    z[e] = __expf(z[e] - from);
    total += z[e];
  }
  total += __shfl_xor(total, 16, 64);
  total += __shfl_xor(total, 32, 64);
  if (i >= o.rows || strip >= o.across) return;
  if (lane < 16) o.strips[i * o.across + strip] = XentStrip{top, total};
  typedef typename XentKept<T>::type K;
  typedef K k4 __attribute__((ext_vector_type(4)));
  if (o.exps && c < o.cols) *reinterpret_cast<k4*>(o.exps + i * o.ldexps + c) = k4{(K)z[0], (K)z[1], (K)z[2], (K)z[3]};
}

// lse and loss of a row from its strips, by LANES lanes.  Bytes bound it (8192 rows of 2048 strips 60 us), few rows its one pass (4 us).
template <int LANES>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void xent_join_kernel(const XentStrip* __restrict__ strips, const int64_t across,
                                                                              float* __restrict__ picked, const XentTargets t, const int64_t rows,
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
    // the loss from the difference of the logits: of a row that is sure of its target, lse's rounding would be more than is left of it
    const float l = logf(all.sum);
    if (lse) lse[row] = all.top + l;
    if (xent_target(t, row) >= 0) {
      const float v = (all.top - picked[row]) + l;
      picked[row] = v;
      if (loss) loss[row] = v;
    } else if (loss) loss[row] = 0.0f;
  }
}

// The sum or mean of the losses of the rows that count, and what each of them has of it.  One workgroup, whose loads bound it: 4096 rows 4 us, 8192
// 6.5, a million 590, beside products of milliseconds.
__global__ __launch_bounds__(1024) void xent_reduce_kernel(const float* __restrict__ loss, const XentTargets t, const int64_t rows, const bool mean,
                                                           float* __restrict__ out, float* __restrict__ weights) {
  constexpr int EACH = 4;
  __shared__ float sums[16];
  __shared__ int counts[16];
  float sum = 0.0f;
  int count = 0;
  for (int64_t i0 = threadIdx.x; i0 < rows; i0 += 1024 * EACH) {
    int64_t raw[EACH];
    float v[EACH];
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const int64_t i = i0 + 1024 * e;
      raw[e] = xent_raw(t, i < rows ? i : rows - 1);
      v[e] = i < rows ? loss[i] : 0.0f;
    }
#pragma unroll
    for (int e = 0; e < EACH; ++e)
      if (i0 + 1024 * e < rows && xent_said(t, raw[e]) >= 0) {
        sum += v[e];
        ++count;
      }
  }
#pragma unroll
  for (int off = 1; off < 64; off *= 2) {
    sum += __shfl_xor(sum, off, 64);
    count += __shfl_xor(count, off, 64);
  }
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum, counts[threadIdx.x >> 6] = count;
  __syncthreads();
  sum = sums[0], count = counts[0];
#pragma unroll
  for (int w = 1; w < 16; ++w) sum += sums[w], count += counts[w];
  if (threadIdx.x == 0) *out = mean ? sum / (float)count : sum;
  if (!weights) return;
  const float weight = mean ? 1.0f / (float)count : 1.0f;
  for (int64_t i = threadIdx.x; i < rows; i += 1024) weights[i] = xent_target(t, i) >= 0 ? weight : 0.0f;
}

// ---------------------------------------------------------------------------
// The gradient.
// ---------------------------------------------------------------------------

// What e is multiplied by, and the products with it.
struct XentScale {
  float up, down;
};

// For operands in 16 bits: the largest |g| of a row that counts comes to 1, in fp16 to 2^14.
template <typename T>
__global__ __launch_bounds__(1024) void xent_scale_kernel(const float* __restrict__ g, const XentTargets t, const int64_t rows, XentScale* scale) {
  constexpr int EACH = 4;
  constexpr float TOP = std::is_same<T, _Float16>::value ? 16384.0f : 1.0f;
  __shared__ float part[16];
  float most = 0.0f;
  for (int64_t i0 = threadIdx.x; i0 < rows; i0 += 1024 * EACH) {
    int64_t raw[EACH];
    float v[EACH];
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const int64_t i = i0 + 1024 * e < rows ? i0 + 1024 * e : rows - 1;
      raw[e] = xent_raw(t, i);
      v[e] = g[i];
    }
#pragma unroll
    for (int e = 0; e < EACH; ++e)
      if (xent_said(t, raw[e]) >= 0) most = fmaxf(most, fabsf(v[e]));
  }
#pragma unroll
  for (int off = 1; off < 64; off *= 2) most = fmaxf(most, __shfl_xor(most, off, 64));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = most;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 16; ++w) most = fmaxf(most, part[w]);
    *scale = XentScale{1.0f, 1.0f};
    if (most > 0.0f && most < INFINITY) {
      most = fmaxf(most, 0x1p-100f);
      if (TOP == 1.0f) most = fminf(most, 0x1p126f);           // its reciprocal stays a normal number
      *scale = XentScale{TOP / most, most / TOP};
    }
  }
}

// x with zeros in the rows that do not count (without targets: all do) and behind every row's end, rows on 16 bytes.
template <typename T>
__global__ __launch_bounds__(256) void xent_rows_kernel(const T* __restrict__ x, const int64_t ldx, const XentTargets t, const int64_t rows,
                                                        const int64_t k, T* __restrict__ to, const int64_t ldto, const int64_t first) {
  typedef typename Core<T>::piece_t piece_t;
  const int64_t across = ldto / Core<T>::VEC, id = (first + blockIdx.x) * 256 + threadIdx.x, i = id / across, c = (id - i * across) * Core<T>::VEC;
  if (i >= rows) return;
  piece_t v = {};
  if (!t.target || xent_target(t, i) >= 0) v = row_piece<T>(x + i * ldx, c, k);
  *reinterpret_cast<piece_t*>(to + i * ldto + c) = v;
}

template <typename T>
struct XentSlope {
  XentTargets t;
  const T* bias;                       // null: none
  const float *lse, *g;
  const float* loss;                   // null: the target's e from lse, as precise as that is
  const XentScale* scale;              // null: 1
  T* e;                                // rows x lde, columns from `first` on; then its other parts, likewise
  int64_t lde;
  float* sums;                         // parts x cols of db; null: not wanted
  int64_t rows, cols, first;           // of the piece
};

// What a row needs for its e: its weight (zero if it does not count; NaN where lse is no number, as all of its e), its target, counted from column
// `from` on.
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
  const float lse = o.lse[i];
  return XentRow{lse, o.g[i] + (lse - lse), true, t - o.first - from};
}

// Tiles of e.  PARTS: numbers of type T that add up to an element of it.  As the forward pass's, with the stores of e (4096 x 1024 over 50003 words bf16 450 to 515 us).
template <typename T, typename S, bool DIRECT, int PARTS>
__global__ __launch_bounds__(S::THREADS) void xent_slope_kernel(const Operand<T> r, const Operand<T> c, const XentSlope<T> o, const XentUnits u) {
  typedef typename Core<T>::acc_t acc_t;
  typedef T t4 __attribute__((ext_vector_type(4)));
  constexpr int STRIP = S::TN * 16;
  __shared__ __attribute__((aligned(16))) char lds[S::NB * S::SLAB];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int wrow = wave / S::WN * (S::TM * 16) + (lane & 15), quad = 4 * (lane >> 4);
  const float up = o.scale ? o.scale->up : 1.0f, down = o.scale ? o.scale->down : 1.0f;
  float lse[S::TM], g[S::TM];
  int at[S::TM];                       // -1: no target among this lane's columns; -2: the row does not count
  auto early = [&](const XentUnit& x) {
    const int64_t first = ((int64_t)x.bj * S::WN + wave % S::WN) * STRIP + quad;
#pragma unroll
    for (int b = 0; b < S::TM; ++b) {
      const XentRow row = xent_row(o, (int64_t)x.bi * S::BM + wrow + 16 * b, first);
      lse[b] = row.lse;
      g[b] = row.g;
      at[b] = !row.counts ? -2 : row.target >= 0 && row.target < STRIP ? (int)row.target : -1;
    }
  };
  xent_units<T, S, false, false, DIRECT>(lds, r, c, u, early, [&](const XentUnit& x, acc_t (&acc)[S::TN][S::TM]) {
    const int64_t row0 = (int64_t)x.bi * S::BM + wrow, col0 = ((int64_t)x.bj * S::WN + wave % S::WN) * STRIP;
    if (o.bias) {
#pragma unroll
      for (int a = 0; a < S::TN; ++a)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int64_t j = col0 + quad + 16 * a + e;
          const float add = j < o.cols ? (float)o.bias[j] : 0.0f;
#pragma unroll
          for (int b = 0; b < S::TM; ++b) acc[a][b][e] += add;
        }
    }
#pragma unroll
    for (int b = 0; b < S::TM; ++b) {
      const float weight = g[b] * up;
      // no logit is above lse, but for sums in another order than the forward pass's, which at 1e10 may differ by a thousand
#pragma unroll
      for (int a = 0; a < S::TN; ++a)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[a][b][e] = __expf(fminf(acc[a][b][e] - lse[b], 0.0f));
      if (__any(at[b] >= 0)) {         // of few strips of a large vocabulary
        const float own = o.loss && at[b] >= 0 ? expm1f(-o.loss[row0 + 16 * b]) : 0.0f;
#pragma unroll
        for (int a = 0; a < S::TN; ++a)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (at[b] == 16 * a + e) acc[a][b][e] = o.loss ? own : acc[a][b][e] - 1.0f;
      }
#pragma unroll
      for (int a = 0; a < S::TN; ++a) acc[a][b] *= weight;
      if (__any(at[b] == -2)) {        // their logits may be anything
#pragma unroll
        for (int a = 0; a < S::TN; ++a)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[a][b][e] = at[b] == -2 ? 0.0f : acc[a][b][e];
      }
    }
    if (o.sums) {
      const int64_t part = (int64_t)x.bi * S::WM + wave / S::WN;
#pragma unroll
      for (int a = 0; a < S::TN; ++a)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float s = 0.0f;
#pragma unroll
          for (int b = 0; b < S::TM; ++b) s += acc[a][b][e];
#pragma unroll
          for (int off = 1; off < 16; off *= 2) s += __shfl_xor(s, off, 64);
          const int64_t j = col0 + quad + 16 * a + e;
          if ((lane & 15) == 0 && j < o.cols) o.sums[part * o.cols + j] = s * down;
        }
    }
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
#pragma unroll
      for (int b = 0; b < S::TM; ++b) {
        const int64_t i = row0 + 16 * b;
        // rows of e are whole pieces of 16 bytes long
        xent_store<T, S::TN>(o.e + (part * o.rows + i) * o.lde, col0, o.cols, i < o.rows, [&](const int a) {
          const t4 v = t4{(T)acc[a][b][0], (T)acc[a][b][1], (T)acc[a][b][2], (T)acc[a][b][3]};
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (PARTS > 1) acc[a][b][e] -= (float)v[e];                  // what is left for the next part
          return v;
        });
      }
    }
  });
}

// e from what the forward pass kept: 16 XENT_EACH rows of 16 pieces by a workgroup, as in the gradient of the activation.  Bytes bound it: 8192 rows
// over 65536 words 424 us (2.1 GB, 5.1 TB/s), where forming z again takes 3500.
constexpr int XENT_EACH = 4;

template <typename T>
__global__ __launch_bounds__(256) void xent_slope_kept_kernel(const XentSlope<T> o, const typename XentKept<T>::type* __restrict__ exps,
                                                              const int64_t ldexps,
                                                              const XentStrip* __restrict__ strips, const int64_t across, const int64_t strip,
                                                              const int64_t first) {
  typedef typename Core<T>::piece_t piece_t;
  constexpr int VEC = Core<T>::VEC;
  __shared__ float part[16][16 * VEC];
  const int64_t wide = (o.cols + 16 * VEC - 1) / (16 * VEC), id = first + blockIdx.x, down = id / wide;
  const int t = threadIdx.x / 16, c = threadIdx.x % 16 * VEC;
  const int64_t col0 = (id - down * wide) * (16 * VEC), col = col0 + c, row = down * (16 * XENT_EACH) + t;
  const bool there = col < o.cols;
  const float up = o.scale ? o.scale->up : 1.0f;
  typedef typename XentKept<T>::type kept_t __attribute__((ext_vector_type(VEC)));
  kept_t x[XENT_EACH];
  XentRow of[XENT_EACH];
  float top[XENT_EACH], loss[XENT_EACH];
#pragma unroll
  for (int r = 0; r < XENT_EACH; ++r) {
    const int64_t i = row + 16 * r;
    of[r] = xent_row(o, i, col);
    x[r] = kept_t{};
    top[r] = loss[r] = 0.0f;
    if (of[r].counts && there) {
      x[r] = *reinterpret_cast<const kept_t*>(exps + i * ldexps + o.first + col);
      top[r] = strips[i * across + (o.first + col) / strip].top;
      loss[r] = o.loss[i];
    }
  }
  float sum[VEC] = {};
#pragma unroll
  for (int r = 0; r < XENT_EACH; ++r) {
    const int64_t i = row + 16 * r;
    // of a strip of nothing but -inf, whose exponentials are zero, beside finite logits of any size
    const float share = top[r] == -INFINITY ? 1.0f : __expf(top[r] - of[r].lse);
    const float own = expm1f(-loss[r]);
    piece_t d;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float p = (float)x[r][e] * share;
      const float q = of[r].target == e ? own : p;
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
  bool vec;                            // eight (fp32: four) elements of a row can be moved at once
};

// Four neighbours of a row from column j on: with what the pieces before came to.
template <typename O>
__device__ __forceinline__ void xent_sum(const XentOut<O>& o, const int64_t i, const int64_t j, const float down, float (&v)[4]) {
  const float* const total = o.total + i * o.cols + j;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[e] *= down;
    if (!o.begins && i < o.rows && j + e < o.cols) v[e] += total[e];
  }
}
template <typename O>
__device__ __forceinline__ void xent_put(const XentOut<O>& o, const int64_t i, const int64_t j, const float (&v)[4]) {
  typedef O o4 __attribute__((ext_vector_type(4)));
  if (i >= o.rows) return;
  if (o.ends && o.vec && j + 4 <= o.cols) {
    *reinterpret_cast<o4*>(o.y + i * o.ldy + j) = o4{(O)v[0], (O)v[1], (O)v[2], (O)v[3]};
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (j + e < o.cols) {
      if (o.ends) o.y[i * o.ldy + j + e] = (O)v[e];
      else o.total[i * o.cols + j + e] = v[e];
    }
}

// dx = e W (C outer) and dW = e^T x (both outer).  The matrix cores bound them: 8192 x 65536 x 4096 bf16 3.36 ms (1.31 PFLOP/s, the library's 1.31)
// and 3.53 (1.25, 1.14); 4096 x 50003 x 1024 357 and 395 us: dx's 64 tiles by four workgroups each (976 as tiles of 64, unsplit).
template <typename T, typename O, typename S, bool ROUTER, bool DIRECT>
__global__ __launch_bounds__(S::THREADS) void xent_product_kernel(const Operand<T> r, const Operand<T> c, const XentOut<O> o, const XentUnits u) {
  typedef typename Core<T>::acc_t acc_t;
  typedef O o4 __attribute__((ext_vector_type(4)));
  __shared__ __attribute__((aligned(16))) char lds[S::NB * S::SLAB];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), quad = 4 * (lane >> 4);
  const int wrow = wave / S::WN * (S::TM * 16) + (lane & 15), wcol = wave % S::WN * (S::TN * 16);
  const float down = o.scale ? o.scale->down : 1.0f;
  xent_units<T, S, ROUTER, true, DIRECT>(lds, r, c, u, [](const XentUnit&) {}, [&](const XentUnit& x, acc_t (&acc)[S::TN][S::TM]) {
    if (x.part >= 0) {
      float* const to = u.parts + (int64_t)x.part * (S::BM * S::BN) + wcol + quad;
#pragma unroll
      for (int b = 0; b < S::TM; ++b)
#pragma unroll
        for (int a = 0; a < S::TN; ++a) *reinterpret_cast<acc_t*>(to + (wrow + 16 * b) * S::BN + 16 * a) = acc[a][b];
      return;
    }
    const int64_t row0 = (int64_t)x.bi * S::BM + wrow, col0 = (int64_t)x.bj * S::BN + wcol;
#pragma unroll
    for (int b = 0; b < S::TM; ++b) {
      const int64_t i = row0 + 16 * b;
#pragma unroll
      for (int a = 0; a < S::TN; a += 2) {
        float v[2][4];
#pragma unroll
        for (int h = 0; h < 2 && a + h < S::TN; ++h) {
#pragma unroll
          for (int e = 0; e < 4; ++e) v[h][e] = acc[a + h][b][e];
          xent_sum(o, i, col0 + 16 * (a + h) + quad, down, v[h]);
        }
        if constexpr (sizeof(O) == 2 && S::TN % 2 == 0) {
          const int64_t j = col0 + 16 * a;
          if (o.ends && o.vec && j + 32 <= o.cols) {
            const auto w = XentEight<O>::of(o4{(O)v[0][0], (O)v[0][1], (O)v[0][2], (O)v[0][3]}, o4{(O)v[1][0], (O)v[1][1], (O)v[1][2], (O)v[1][3]});
            if (i < o.rows) *reinterpret_cast<typename XentEight<O>::eight_t*>(o.y + i * o.ldy + j + XentEight<O>::col()) = w;
            continue;
          }
        }
#pragma unroll
        for (int h = 0; h < 2 && a + h < S::TN; ++h) xent_put(o, i, col0 + 16 * (a + h) + quad, v[h]);
      }
    }
  });
}

// The parts of the tiles that were shared, added in their order: four neighbours of a row by a thread.
template <typename O, int BM, int BN>
__global__ __launch_bounds__(256) void xent_product_join_kernel(const XentOut<O> o, const XentUnits u) {
  typedef float f4 __attribute__((ext_vector_type(4)));
  constexpr int EACH = BM * BN / 1024;
  const int tile = blockIdx.x / EACH, at = (int)(blockIdx.x % EACH * 256 + threadIdx.x) * 4;
  int bi, bj;
  xent_place(u, u.whole + tile, bi, bj);
  const int64_t i = (int64_t)bi * BM + at / BN, j = (int64_t)bj * BN + at % BN;
  if (i >= o.rows || j >= o.cols) return;
  f4 sum = {};
  for (int s = 0; s < u.splits; ++s) sum += *reinterpret_cast<const f4*>(u.parts + ((int64_t)tile * u.splits + s) * (BM * BN) + at);
  float v[4] = {sum[0], sum[1], sum[2], sum[3]};
  xent_sum(o, i, j, o.scale ? o.scale->down : 1.0f, v);
  xent_put(o, i, j, v);
}

}  // namespace mdet
