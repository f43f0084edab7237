// Matrix products D[i][j] = sum_k R[i][k] C[j][k] on the matrix cores, for the linear layer, its gradient and the
// Gram matrix of a network's Jacobian.  R is the row operand (its index runs along the rows of D), C the column operand.
//
// Pieces.  Every operand is handled in pieces of 16 bytes along k: 8 elements in 16 bits, 4 in fp32, 2 in fp64.  A slab
// is eight pieces (128 bytes) of k.  Lane l of a wavefront supplies piece l / 16 of row l % 16 to a product, which takes
// the four pieces of one half slab at once: one instruction of 16 x 16 x 32 in 16 bits, four of 16 x 16 x 4 in fp32, two
// in fp64 (the e-th elements of the four pieces form the e-th of them; any assignment of k's is valid as long as R and C
// use the same one).  Sums are fp32 for operands in 16 and 32 bits, fp64 for fp64.
//
// The column operand goes in as the instruction's first, so that a lane's four results are neighbours in a row of D
// (fp64: four columns apart) and leave in one store.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mdet {

constexpr int GEMM_PIECES = 8;        // pieces of a slab

template <typename T> struct Core;

template <> struct Core<__bf16> {
  typedef float acc1_t;
  typedef float acc_t __attribute__((ext_vector_type(4)));
  typedef __bf16 piece_t __attribute__((ext_vector_type(8)));
  static constexpr int VEC = 8;
  static __device__ __forceinline__ void mma(const piece_t& c, const piece_t& r, acc_t& acc) {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(c, r, acc, 0, 0, 0);
  }
  static __device__ __forceinline__ int col(int lane, int e) { return 4 * (lane >> 4) + e; }
};

template <> struct Core<_Float16> {
  typedef float acc1_t;
  typedef float acc_t __attribute__((ext_vector_type(4)));
  typedef _Float16 piece_t __attribute__((ext_vector_type(8)));
  static constexpr int VEC = 8;
  static __device__ __forceinline__ void mma(const piece_t& c, const piece_t& r, acc_t& acc) {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(c, r, acc, 0, 0, 0);
  }
  static __device__ __forceinline__ int col(int lane, int e) { return 4 * (lane >> 4) + e; }
};

template <> struct Core<float> {
  typedef float acc1_t;
  typedef float acc_t __attribute__((ext_vector_type(4)));
  typedef float piece_t __attribute__((ext_vector_type(4)));
  static constexpr int VEC = 4;
  static __device__ __forceinline__ void mma(const piece_t& c, const piece_t& r, acc_t& acc) {
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(c[e], r[e], acc, 0, 0, 0);
  }
  static __device__ __forceinline__ int col(int lane, int e) { return 4 * (lane >> 4) + e; }
};

template <> struct Core<double> {
  typedef double acc1_t;
  typedef double acc_t __attribute__((ext_vector_type(4)));
  typedef double piece_t __attribute__((ext_vector_type(2)));
  static constexpr int VEC = 2;
  static __device__ __forceinline__ void mma(const piece_t& c, const piece_t& r, acc_t& acc) {
#pragma unroll
    for (int e = 0; e < 2; ++e) acc = __builtin_amdgcn_mfma_f64_16x16x4f64(c[e], r[e], acc, 0, 0, 0);
  }
  static __device__ __forceinline__ int col(int lane, int e) { return 4 * e + (lane >> 4); }
};

// Element (i, k) stands at p[i * stride + k], or, with k outer, at p[k * stride + i].
template <typename T>
struct Operand {
  const T* p;
  int64_t stride;
  int64_t rows;                        // i < rows
};

// ---------------------------------------------------------------------------
// The staged tile: BM x BN of D by WM x WN wavefronts, slabs of both operands double buffered in LDS.
//
// A slab of B rows takes 128 B bytes of LDS.  With k inner, row i's eight pieces stand in the order piece ^ (i & 7): the
// eight lanes that one LDS cycle serves read one piece of eight rows, from eight different places.  With k outer, the slab
// lies as it does in memory, row k's elements side by side: in 16 bits the transposing read hands lane l the four k's of
// column l % 16 out of four rows of 32 bytes, in fp32 the instructions take single elements.  There the blocks of 16
// columns of row k stand in the order block ^ f(k), so that the rows read together lie in different banks.
//
// DIRECT: memory goes straight into LDS (every lane names the 16 bytes that land at its place), for operands whose rows
// start on 16 bytes.  Otherwise, and for the ragged last slab, pieces pass through registers, whole ones in one load of
// any alignment, those that hang over an edge element by element.
// ---------------------------------------------------------------------------
typedef __attribute__((address_space(3))) char* gemm_lds_ptr;

// 16 bytes a lane from base + off (base the same in all lanes) to LDS, lane by lane from byte `at` on.  Written out because
// the compiler, told of the load, waits for it in front of the next read of anything in LDS; the caller waits for it by
// itself (s_waitcnt vmcnt).
__device__ __forceinline__ void gemm_to_lds(const char* base, const unsigned off, const unsigned at) {
  const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)base);
  const unsigned hi = __builtin_amdgcn_readfirstlane((unsigned)((uintptr_t)base >> 32));
  const unsigned long long from = ((unsigned long long)hi << 32) | lo;
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"{m0}"(at), "v"(off), "s"(from));
}

// All of a wavefront's loads and LDS accesses are done, and behind the barrier those of all.
__device__ __forceinline__ void gemm_landed() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

template <int BM_, int BN_, int WM_, int WN_>
struct Tile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
  static constexpr int WAVES = WM * WN, THREADS = 64 * WAVES;
  static constexpr int TM = BM / WM / 16, TN = BN / WN / 16;   // 16 x 16 parts of a wavefront, down and across
  static constexpr int SLAB = 128 * (BM + BN);                 // bytes of one slab of both operands
};

// Staging of an operand: B rows of it from i0 on.
template <typename T, int B, int WAVES, bool OUTER, bool DIRECT>
struct Stage {
  typedef typename Core<T>::piece_t piece_t;
  static constexpr int VEC = Core<T>::VEC, BK = GEMM_PIECES * VEC;
  static constexpr int NP = B * GEMM_PIECES / (64 * WAVES);    // pieces a lane brings of a slab
  static constexpr int PR = B / VEC;                           // k outer: pieces of a row k
  static_assert(NP * 64 * WAVES == B * GEMM_PIECES, "whole pieces");

  const T* p;
  int64_t stride, rows, i0;
  unsigned off[DIRECT ? NP : 1];
  piece_t held[NP];

  // Order of the blocks of 16 columns of row k.
  static __device__ __forceinline__ int swizzle(const int k) {
    if constexpr (sizeof(T) == 2) return ((k & 3) | ((k >> 1) & 4)) & (B / 16 - 1);
    else return (k >> 2) & 3;
  }
  // Row and k of the piece that stands at place `id` of the slab.
  static __device__ __forceinline__ void piece_at(const int id, int& row, int& k) {
    if constexpr (OUTER) {
      constexpr int PB = 16 / VEC;                             // pieces of a block of 16 columns
      k = id / PR;
      const int at = id % PR;
      row = (((at / PB) ^ swizzle(k)) * PB + at % PB) * VEC;
    } else {
      row = id / GEMM_PIECES;
      k = ((id % GEMM_PIECES) ^ (row & 7)) * VEC;
    }
  }
  static __device__ __forceinline__ int place(const int v) {
    return (v * WAVES + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6)) * 64 + ((int)threadIdx.x & 63);
  }

  __device__ __forceinline__ Stage(const Operand<T>& o, const int64_t first) : p(o.p), stride(o.stride), rows(o.rows), i0(first) {
    if constexpr (DIRECT) {
#pragma unroll
      for (int v = 0; v < NP; ++v) {
        int row, k;
        piece_at(place(v), row, k);
        // rows behind the last are not stored: any memory of the operand will do for them
        if (OUTER) {
          const int64_t i = i0 + row > rows - VEC ? rows - VEC : i0 + row;
          off[v] = (unsigned)((k * stride + (i - i0)) * (int64_t)sizeof(T));
        } else {
          const int64_t i = i0 + row > rows - 1 ? rows - 1 : i0 + row;
          off[v] = (unsigned)(((i - i0) * stride + k) * (int64_t)sizeof(T));
        }
      }
    }
  }
  // The slab from k on straight to LDS at byte `at`.
  __device__ __forceinline__ void direct(const int64_t k, const unsigned at) const {
    const char* const base = reinterpret_cast<const char*>(OUTER ? p + k * stride + i0 : p + i0 * stride + k);
#pragma unroll
    for (int v = 0; v < NP; ++v) gemm_to_lds(base, off[v], at + 16u * (unsigned)(place(v) & ~63));
  }
  // The slab from k on into registers; what lies outside of the operand is zero.
  __device__ __forceinline__ void load(const int64_t k0, const int64_t kend) {
#pragma unroll
    for (int v = 0; v < NP; ++v) {
      int row, kk;
      piece_at(place(v), row, kk);
      const int64_t i = i0 + row, k = k0 + kk;
      const int64_t left = OUTER ? (k < kend ? rows - i : 0) : (i < rows ? kend - k : 0);   // elements that there are
      const T* const from = OUTER ? p + k * stride + i : p + i * stride + k;
      piece_t x = {};
      if (left >= VEC) __builtin_memcpy(&x, from, 16);
      else {
#pragma unroll
        for (int e = 0; e < VEC - 1; ++e)
          if (e < left) x[e] = from[e];
      }
      held[v] = x;
    }
  }
  __device__ __forceinline__ void put(char* const lds) const {
#pragma unroll
    for (int v = 0; v < NP; ++v) *reinterpret_cast<piece_t*>(lds + 16 * place(v)) = held[v];
  }
  // Rows 16 t + lane % 16, piece 4 h + lane / 16: what the lane supplies to a product.
  static __device__ __forceinline__ piece_t fragment(const char* const lds, const int t, const int h) {
    const int lane = threadIdx.x & 63, g = lane >> 4, j = lane & 15;
    if constexpr (!OUTER) {
      return *reinterpret_cast<const piece_t*>(lds + (16 * t + j) * 128 + (((4 * h + g) ^ (j & 7)) << 4));
    } else if constexpr (sizeof(T) == 2) {
      typedef short half_t __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) half_t* lds_half_ptr;
      typedef short whole_t __attribute__((ext_vector_type(8)));
      const int k = 32 * h + 8 * g + (j >> 2);
      const char* const at = lds + k * (B * 2) + ((t ^ swizzle(k)) << 5) + ((j & 3) << 3);
      const half_t low = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_half_ptr)(at));
      const half_t high = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_half_ptr)(at + 4 * (B * 2)));
      const whole_t both = __builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7);
      return __builtin_bit_cast(piece_t, both);
    } else {
      piece_t x;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const int k = 4 * VEC * h + VEC * g + e;
        x[e] = *reinterpret_cast<const T*>(lds + k * (B * (int)sizeof(T)) + ((t ^ swizzle(k)) << 6) + (j << 2));
      }
      return x;
    }
  }
};

// acc[a][b] += columns 16 a .. times rows 16 b .. of this wavefront's part of the tile at (row0, col0), over k0 .. kend - 1.
// `lds`: 2 * Tile::SLAB bytes, which are not read any more when the last wavefront returns.
template <typename T, typename S, bool ROUTER, bool COUTER, bool DIRECT>
__device__ __forceinline__ void tile_accumulate(typename Core<T>::acc_t (&acc)[S::TN][S::TM], char* const lds, const Operand<T>& r,
                                                const Operand<T>& c, const int64_t row0, const int64_t col0, const int64_t k0,
                                                const int64_t kend) {
  typedef Stage<T, S::BM, S::WAVES, ROUTER, DIRECT> RS;
  typedef Stage<T, S::BN, S::WAVES, COUTER, DIRECT> CS;
  constexpr int BK = RS::BK;
  RS rs(r, row0);
  CS cs(c, col0);
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int wr = wave / S::WN * S::TM, wc = wave % S::WN * S::TN;      // first 16 x 16 part of this wavefront
  const unsigned lds0 = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(gemm_lds_ptr)lds);
  const int slabs = (int)((kend - k0 + BK - 1) / BK);
  // brings slab s: straight to LDS where it is whole, otherwise into registers
  auto bring = [&](const int s) {
    const int64_t k = k0 + (int64_t)s * BK;
    if (DIRECT && k + BK <= kend) {
      rs.direct(k, lds0 + (s & 1) * S::SLAB);
      cs.direct(k, lds0 + (s & 1) * S::SLAB + 128 * S::BM);
      return false;
    }
    rs.load(k, kend);
    cs.load(k, kend);
    return true;
  };
  auto put = [&](const int s) {
    rs.put(lds + (s & 1) * S::SLAB);
    cs.put(lds + (s & 1) * S::SLAB + 128 * S::BM);
  };
  if (slabs > 0 && bring(0)) put(0);
  for (int s = 0; s < slabs; ++s) {
    gemm_landed();
    const bool held = s + 1 < slabs && bring(s + 1);
    const char* const at = lds + (s & 1) * S::SLAB;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      typename Core<T>::piece_t cf[S::TN], rf[S::TM];
#pragma unroll
      for (int a = 0; a < S::TN; ++a) cf[a] = CS::fragment(at + 128 * S::BM, wc + a, h);
#pragma unroll
      for (int b = 0; b < S::TM; ++b) rf[b] = RS::fragment(at, wr + b, h);
#pragma unroll
      for (int b = 0; b < S::TM; ++b)
#pragma unroll
        for (int a = 0; a < S::TN; ++a) Core<T>::mma(cf[a], rf[b], acc[a][b]);
    }
    if (held) put(s + 1);
  }
}

// f(a, b, e, row, column of the tile) for each element e of acc[a][b] that this lane holds.
template <typename T, typename S, typename F>
__device__ __forceinline__ void tile_each(F&& f) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
#pragma unroll
  for (int b = 0; b < S::TM; ++b)
#pragma unroll
    for (int a = 0; a < S::TN; ++a)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        f(a, b, e, (wave / S::WN * S::TM + b) * 16 + (lane & 15), (wave % S::WN * S::TN + a) * 16 + Core<T>::col(lane, e));
}

// Whether an operand's pieces can go straight to LDS: rows on 16 bytes (with k outer their number a whole number of
// pieces), offsets within a slab in 32 bits.
template <typename T, bool OUTER, int B>
bool gemm_straight(const Operand<T>& o, const int64_t k) {
  const int64_t bytes = o.stride * (int64_t)sizeof(T), lines = OUTER ? k : o.rows;
  return (uintptr_t)o.p % 16 == 0 && (lines == 1 || bytes % 16 == 0) && (!OUTER || o.rows % Core<T>::VEC == 0) &&
         bytes < (int64_t(1) << 31) / (B > 64 ? B : 64);
}

// Tile number of workgroup `id` of a launch of 8 ceil(total / 8): workgroups go round the eight chiplets, each of which gets
// a run of consecutive tiles, so that what one L2 holds is read by neighbours.  -1: none.
__device__ __forceinline__ int64_t gemm_tile_number(const int64_t id, const int64_t total) {
  const int64_t per = (total + 7) / 8, t = (id & 7) * per + (id >> 3);
  return (id >> 3) < per && t < total ? t : -1;
}
// Row and column of tile t: eight rows of tiles at a time, column by column.
__device__ __forceinline__ void gemm_tile_place(const int64_t t, const int64_t down, const int64_t across, int64_t& bi, int64_t& bj) {
  const int64_t group = t / (8 * across), in = t - group * 8 * across, left = down - 8 * group, rows = left < 8 ? left : 8;
  bi = 8 * group + in % rows;
  bj = in / rows;
}

}  // namespace mdet
