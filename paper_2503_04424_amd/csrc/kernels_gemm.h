// Matrix products D[i][j] = sum_k R[i][k] C[j][k] on the matrix cores, for the linear layer, its gradient and the
// Gram matrix of a network's Jacobian.  R is the row operand (its index runs along the rows of D), C the column operand.
//
// Pieces.  Every operand is handled in pieces of 16 bytes along k: 8 elements in 16 bits, 4 in fp32, 2 in fp64.  A slab
// is eight pieces (128 bytes) of k.  Lane l of a wavefront supplies piece l / 16 of row l % 16 to a product, which takes
// four pieces at once: one instruction of 16 x 16 x 32 in 16 bits, four of 16 x 16 x 4 in fp32, two
// in fp64 (the e-th elements of the four pieces form the e-th of them; any assignment of k's is valid as long as R and C
// use the same one).  Sums are fp32 for operands in 16 and 32 bits, fp64 for fp64.
//
// The column operand goes in as the instruction's first, so that a lane's four results are neighbours in a row of D
// (fp64: four columns apart) and leave in one store.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace mdet {

constexpr int PIECES = 8;              // of a slab, along k

template <typename T> struct Core;

template <> struct Core<__bf16> {
  typedef float acc1_t;
  typedef float acc_t __attribute__((ext_vector_type(4)));
  typedef __bf16 piece_t __attribute__((ext_vector_type(8)));
  static constexpr int VEC = 8;
  static __device__ __forceinline__ void mma(const piece_t& c, const piece_t& r, acc_t& acc) {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(c, r, acc, 0, 0, 0);
  }
  // Two products into two accumulators, in turn: neither waits for the one before it.
  static __device__ __forceinline__ void mma_two(const piece_t (&c)[2], const piece_t (&r)[2], acc_t& acc, acc_t& other) {
    mma(c[0], r[0], acc);
    mma(c[1], r[1], other);
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
  static __device__ __forceinline__ void mma_two(const piece_t (&c)[2], const piece_t (&r)[2], acc_t& acc, acc_t& other) {
    mma(c[0], r[0], acc);
    mma(c[1], r[1], other);
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
  static __device__ __forceinline__ void mma_two(const piece_t (&c)[2], const piece_t (&r)[2], acc_t& acc, acc_t& other) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      acc = __builtin_amdgcn_mfma_f32_16x16x4f32(c[0][e], r[0][e], acc, 0, 0, 0);
      other = __builtin_amdgcn_mfma_f32_16x16x4f32(c[1][e], r[1][e], other, 0, 0, 0);
    }
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
  static __device__ __forceinline__ void mma_two(const piece_t (&c)[2], const piece_t (&r)[2], acc_t& acc, acc_t& other) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      acc = __builtin_amdgcn_mfma_f64_16x16x4f64(c[0][e], r[0][e], acc, 0, 0, 0);
      other = __builtin_amdgcn_mfma_f64_16x16x4f64(c[1][e], r[1][e], other, 0, 0, 0);
    }
  }
  static __device__ __forceinline__ int col(int lane, int e) { return 4 * e + (lane >> 4); }
};

// Element (i, k) stands at p[i * stride + k], or, with k outer, at p[k * stride + i].
template <typename T>
struct Operand {
  const T* p;
  int64_t stride;
  int64_t rows;                        // i < rows
  bool near;                           // offsets within a slab fit 32 bits
  bool straight;                       // and its whole slabs can go straight to LDS
};

// ---------------------------------------------------------------------------
// The staged tile: BM x BN of D by WM x WN wavefronts, slabs of both operands in NB buffers in LDS.
//
// With k inner, row i's eight pieces (a line of 128 bytes) stand in the order piece ^ (i & 7): lanes that read one piece of
// consecutive rows read from different places.  With k outer, the slab lies as it does in memory, row k's elements side by
// side: in 16 bits the transposing read hands lane l the four k's of column l % 16 out of four rows of 32 bytes, in fp32 the
// instructions take single elements.  There the blocks of 16 columns of row k stand in the order block ^ f(k), so that the
// rows read together lie in different banks.
//
// DIRECT: memory goes straight into LDS (every lane names the 16 bytes that land at its place), for operands whose rows
// start on 16 bytes.  Otherwise pieces pass through registers, whole ones in one load of any alignment, those that hang
// over an edge element by element, beside the products of the slab before; in a DIRECT product that is done without such an
// overlap, for the ragged last slab and for an operand beside the others that is not straight.
// ---------------------------------------------------------------------------
typedef __attribute__((address_space(3))) char* gemm_lds_ptr;

// A value that is the same in all lanes, in scalar registers whatever the compiler had in mind for it.
template <typename V>
__device__ __forceinline__ V gemm_scalar(const V v) {
  const uint64_t x = (uint64_t)v;
  return (V)(((uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32) | (unsigned)__builtin_amdgcn_readfirstlane((int)x));
}

// 16 bytes a lane from base + off (base the same in all lanes) to LDS, lane by lane from byte `at` on.  Written out because
// the compiler, told of the load, waits for it in front of the next read of anything in LDS; the caller waits for it by
// itself (s_waitcnt vmcnt).  The base may have come out of vector registers a moment ago: a memory instruction has to keep
// five wait states behind a vector instruction that wrote its scalar registers, which the compiler does not see to in here.
__device__ __forceinline__ void gemm_to_lds(const char* base, const unsigned off, const unsigned at) {
  const uint64_t from = gemm_scalar((uint64_t)base);
  asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"{m0}"(at), "v"(off), "s"(from));
}

// All of a wavefront's loads but the last `LATER` and all of its LDS accesses are done, and behind the barrier those of all.
template <int LATER>
__device__ __forceinline__ void gemm_landed() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"i"(LATER) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// All of a wavefront's LDS accesses are done, and behind the barrier those of all; loads into registers go on.
__device__ __forceinline__ void gemm_put_down() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// NB: slabs in LDS.
template <int BM_, int BN_, int WM_, int WN_, int NB_>
struct Tile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NB = NB_;
  static constexpr int WAVES = WM * WN, THREADS = 64 * WAVES;
  static constexpr int TM = BM / WM / 16, TN = BN / WN / 16;   // 16 x 16 parts of a wavefront, down and across
  static constexpr int SLAB = 16 * PIECES * (BM + BN);         // bytes of one slab of both operands
};

// Staging of an operand: B rows of it from i0 on.
template <typename T, int B, int WAVES, bool OUTER, bool DIRECT, int HOLD>
struct Stage {
  typedef typename Core<T>::piece_t piece_t;
  static constexpr int VEC = Core<T>::VEC, BK = PIECES * VEC;
  static constexpr int NP = B * PIECES / (64 * WAVES);         // pieces a lane brings of a slab
  static constexpr int PR = B / VEC;                           // k outer: pieces of a row k
  static_assert(NP * 64 * WAVES == B * PIECES, "whole pieces");

  const T* p;
  int64_t stride, rows, i0;
  unsigned off[NP];                    // bytes from the slab's first element to the pieces
  piece_t held[HOLD][NP];

  // Order of the blocks of 16 columns of row k.
  static __device__ __forceinline__ int swizzle(const int k) {
    if constexpr (sizeof(T) == 2) return ((k & 3) | ((k >> 1) & 4)) & (B / 16 - 1);
    else return (k >> 2) & 3 & (B / 16 - 1);
  }
  // Row and k of the piece that stands at place `id` of the slab.
  static __device__ __forceinline__ void piece_at(const int id, int& row, int& k) {
    if constexpr (OUTER) {
      constexpr int PB = 16 / VEC;                             // pieces of a block of 16 columns
      k = id / PR;
      const int at = id % PR;
      row = (((at / PB) ^ swizzle(k)) * PB + at % PB) * VEC;
    } else {
      row = id / PIECES;
      k = ((id % PIECES) ^ (row & 7)) * VEC;
    }
  }
  static __device__ __forceinline__ int place(const int v) {
    return (v * WAVES + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6)) * 64 + ((int)threadIdx.x & 63);
  }

  // Rows from `first` on, which is one of the operand's: a lane's place is held against the last row from there.
  __device__ __forceinline__ void set(const Operand<T>& o, const int64_t first) {
    p = o.p;
    stride = o.stride;
    rows = o.rows;
    i0 = first;
#pragma unroll
    for (int v = 0; v < NP; ++v) {
      int row, k;
      piece_at(place(v), row, k);
      // rows behind the last are not stored: any memory of the operand will do for them
      const int64_t last = OUTER ? (rows - 1) / VEC * VEC : rows - 1;
      const int64_t i = i0 + row > last ? last - i0 : row;
      off[v] = (unsigned)((OUTER ? k * stride + i : i * stride + k) * (int64_t)sizeof(T));
    }
  }
  // Pieces of rows k < end - spare() are whole in memory: with k outer the last piece of a row k may reach into the rows
  // behind it, and those behind the last one are not the operand's.
  __device__ __forceinline__ int spare() const { return OUTER && rows % VEC ? VEC : 0; }
  __device__ __forceinline__ const char* base(const int64_t k) const {
    return reinterpret_cast<const char*>(OUTER ? p + k * stride + i0 : p + i0 * stride + k);
  }
  // Piece v of the slab at `from` = base(k) straight to LDS, the slab at byte `at`.
  __device__ __forceinline__ void direct(const char* const from, const int v, const unsigned at) const {
    gemm_to_lds(from, off[v], at + 16u * (unsigned)(place(v) & ~63));
  }
  // A whole slab into registers, set `h` of them; `from` = base(k).
  __device__ __forceinline__ void load(const char* const from, const int h) {
#pragma unroll
    for (int v = 0; v < NP; ++v) __builtin_memcpy(&held[h][v], from + off[v], 16);
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
      held[0][v] = x;
    }
  }
  __device__ __forceinline__ void put(char* const lds, const int h) const {
#pragma unroll
    for (int v = 0; v < NP; ++v) *reinterpret_cast<piece_t*>(lds + 16 * place(v)) = held[h][v];
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

// A workgroup's way through one product after another: slabs are brought in their order, NB - 1 ahead of the one that is
// multiplied and past the end of its product.  `lds`: NB * SLAB bytes.
template <typename T, typename S, bool ROUTER, bool COUTER, bool DIRECT>
struct TileStream {
  // slabs in registers: as many as small tiles, which wait for memory, have room for
  static constexpr int HOLD = DIRECT ? 1 : S::BM <= 32 ? 4 : S::BM <= 64 && sizeof(T) < 8 ? 3 : 1;
  typedef Stage<T, S::BM, S::WAVES, ROUTER, DIRECT, HOLD> RS;
  typedef Stage<T, S::BN, S::WAVES, COUTER, DIRECT, HOLD> CS;
  typedef typename Core<T>::piece_t piece_t;
  static constexpr int BK = RS::BK, LOADS = RS::NP + CS::NP;   // loads of a wavefront for a slab
  RS rs;
  CS cs;
  bool rquick, cquick, held;           // whole slabs need no look at their edges
  int64_t k, kend;                     // what is left to be brought of the product that slabs are brought of
  int to, at, ahead;                   // buffers to fill and to multiply next, slabs in between
  char* const lds;
  const unsigned lds0;

  __device__ __forceinline__ explicit TileStream(char* where)
      : held(false), k(0), kend(0), to(0), at(0), ahead(0), lds(where),
        lds0(__builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(gemm_lds_ptr)where)) {}

  // Slabs come from this product from here on: the tile at (row0, col0), k from `from` to `end` - 1.
  __device__ __forceinline__ void set(const Operand<T>& r, const Operand<T>& c, const int64_t row0, const int64_t col0, const int64_t from,
                                      const int64_t end) {
    k = from;
    kend = end;
    rquick = DIRECT ? r.straight : r.near;
    cquick = DIRECT ? c.straight : c.near;
    rs.set(r, row0);
    cs.set(c, col0);
  }
  static __device__ __forceinline__ int slabs(const int64_t from, const int64_t end) { return end > from ? (int)((end - from + BK - 1) / BK) : 0; }

  // The next slab, whatever it needs: straight to LDS where that goes and the slab is whole, otherwise through registers.
  template <typename F>
  __device__ __forceinline__ void bring(F&& next) {
    while (k >= kend)
      if (!next()) return;
    char* const slab = lds + to * S::SLAB;
    if constexpr (DIRECT) {
      const bool rcomes = rquick && k + BK + rs.spare() <= kend, ccomes = cquick && k + BK + cs.spare() <= kend;
      const unsigned place = lds0 + to * S::SLAB;
      if (rcomes) {
#pragma unroll
        for (int v = 0; v < RS::NP; ++v) rs.direct(rs.base(k), v, place);
      } else {
        rs.load(k, kend);
        rs.put(slab, 0);
      }
      if (ccomes) {
#pragma unroll
        for (int v = 0; v < CS::NP; ++v) cs.direct(cs.base(k), v, place + 16 * PIECES * S::BM);
      } else {
        cs.load(k, kend);
        cs.put(slab + 16 * PIECES * S::BM, 0);
      }
      // run() counts loads straight to LDS: where some are missing, none is left to be counted
      if (!(rcomes && ccomes)) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    } else {
      rs.load(k, kend);
      cs.load(k, kend);
      held = true;
    }
    k += BK;
    ++ahead;
    to = to + 1 == S::NB ? 0 : to + 1;
  }
  // What bring() left in registers.
  __device__ __forceinline__ void put() {
    if (!DIRECT && held) {
      char* const slab = lds + (to == 0 ? S::NB - 1 : to - 1) * S::SLAB;
      rs.put(slab, 0);
      cs.put(slab + 16 * PIECES * S::BM, 0);
      held = false;
    }
  }
  // next(): sets the product after the one that has been brought whole; false behind the last.
  template <typename F>
  __device__ __forceinline__ void begin(F&& next) {
#pragma unroll
    for (int i = 0; i < (DIRECT ? S::NB - 1 : 1); ++i) bring(next);
    put();
  }
  // acc[a][b] += columns 16 a .. times rows 16 b .. of this wavefront's part of the tile, over the next `count` slabs.
  template <typename F>
  __device__ __forceinline__ void run(typename Core<T>::acc_t (&acc)[S::TN][S::TM], const int count, F&& next) {
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wr = wave / S::WN * S::TM, wc = wave % S::WN * S::TN;    // first 16 x 16 part of this wavefront
    // A wavefront with a single part would wait for each product and each fragment: its two half slabs go into accumulators
    // of their own, in turn, all fragments fetched in front.
    constexpr bool ONE = S::TM * S::TN == 1;
    typename Core<T>::acc_t other = {};
    auto multiply = [&](const char* const slab, auto&& between) {
      if constexpr (ONE) {
        piece_t cf[2], rf[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          cf[h] = CS::fragment(slab + 16 * PIECES * S::BM, wc, h);
          rf[h] = RS::fragment(slab, wr, h);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) between(h);
        Core<T>::mma_two(cf, rf, acc[0][0], other);
        return;
      }
#pragma unroll
      for (int h = 0; h < PIECES / 4; ++h) {
        piece_t cf[S::TN], rf[S::TM];
#pragma unroll
        for (int a = 0; a < S::TN; ++a) cf[a] = CS::fragment(slab + 16 * PIECES * S::BM, wc + a, h);
#pragma unroll
        for (int b = 0; b < S::TM; ++b) rf[b] = RS::fragment(slab, wr + b, h);
#pragma unroll
        for (int b = 0; b < S::TM; ++b) {
          between(h * S::TM + b);
#pragma unroll
          for (int a = 0; a < S::TN; ++a) Core<T>::mma(cf[a], rf[b], acc[a][b]);
        }
      }
    };
    int left = count;
    {
      // The long stretch, without a branch: every slab brought meanwhile is a whole one of this product.
      const int64_t last = kend - (rs.spare() > cs.spare() ? rs.spare() : cs.spare());
      const int64_t whole = rquick && cquick && k < last ? (last - k) / BK : 0;
      int steady = __builtin_amdgcn_readfirstlane(whole < left - ahead ? (int)whole : left - ahead);
      if (ahead == (DIRECT ? S::NB - 1 : 1) && steady > 0) {
        left -= steady;
        const char *rfrom = rs.base(k), *cfrom = cs.base(k);
        int64_t rstep = rs.base(k + BK) - rfrom, cstep = cs.base(k + BK) - cfrom;
        if constexpr (DIRECT) {
          rfrom = gemm_scalar(rfrom), cfrom = gemm_scalar(cfrom);
          rstep = gemm_scalar(rstep), cstep = gemm_scalar(cstep);
        }
        k += (int64_t)steady * BK;
        auto onward = [&] {
          to = to + 1 == S::NB ? 0 : to + 1;
          at = at + 1 == S::NB ? 0 : at + 1;
        };
        if constexpr (DIRECT) {
          for (; steady > 0; --steady) {
            gemm_landed<(S::NB - 2) * LOADS>();
            const unsigned place = lds0 + to * S::SLAB;
            // The loads of a later slab: all in front of this one's products where both operands are read in 128-byte pieces
            // of rows in 16 bits (8192 x 16384 x 4096 1257 TFLOP/s, spread 1176), which wait longest; one behind each strip of
            // products otherwise (k outer 4096 x 4096 x 8192 1384, in front 1324; fp32 4096^3 142, 139).
            constexpr bool FIRST = sizeof(T) == 2 && !ROUTER && !COUTER;
            constexpr int Q = S::TM * PIECES / 4, EACH = (LOADS + Q - 1) / Q;
            auto pieces = [&](const int from, const int end) {
#pragma unroll
              for (int v = from; v < end; ++v) {
                if (v >= LOADS) break;
                if (v < RS::NP) rs.direct(rfrom, v, place);
                else cs.direct(cfrom, v - RS::NP, place + 16 * PIECES * S::BM);
              }
            };
            if constexpr (FIRST) pieces(0, LOADS);
            multiply(lds + at * S::SLAB, [&](const int q) {
              if constexpr (!FIRST) {
                pieces(q * EACH, (q + 1) * EACH);
                __builtin_amdgcn_sched_barrier(0x107);
              }
            });
            rfrom += rstep;
            cfrom += cstep;
            onward();
          }
        } else {
          // HOLD slabs are in registers or on their way there: one is put into LDS behind each slab that is multiplied.
          auto load = [&](const int h) {
            rs.load(rfrom, h);
            cs.load(cfrom, h);
            rfrom += rstep;
            cfrom += cstep;
          };
#pragma unroll
          for (int h = 0; h < HOLD - 1; ++h)
            if (h < steady) load(h);
          for (int s = 0; s < steady; s += HOLD) {
#pragma unroll
            for (int h = 0; h < HOLD; ++h) {
              if (s + h >= steady) break;
              gemm_put_down();
              if (s + h + HOLD - 1 < steady) load((h + HOLD - 1) % HOLD);
              multiply(lds + at * S::SLAB, [](int) {});
              rs.put(lds + to * S::SLAB, h);
              cs.put(lds + to * S::SLAB + 16 * PIECES * S::BM, h);
              onward();
            }
          }
        }
      }
    }
    for (; left > 0; --left) {
      --ahead;
      if (DIRECT && S::NB > 3 && ahead >= 2) gemm_landed<2 * LOADS>();
      else if (DIRECT && S::NB > 2 && ahead >= 1) gemm_landed<LOADS>();
      else gemm_landed<0>();
      bring(next);
      multiply(lds + at * S::SLAB, [](int) {});
      put();
      at = at + 1 == S::NB ? 0 : at + 1;
    }
    if constexpr (ONE) acc[0][0] += other;
  }

  // The same for a wavefront's part of 128 x 64 in 16 bits, with every fragment on its way while others are multiplied: a slab's products are 16
  // steps (of 16 rows and half a slab each), a step's row fragment is fetched three steps ahead, the column fragments a few steps ahead of
  // their half.  Behind step 13 everything of a slab is in registers: the next one has landed by then, its first fragments come in
  // beside the last two steps, and its place in LDS is free for the one after it.  The same sums in the same order as run().  (Cross entropy of 8192 x 4096 over 131072
  // words in bf16: 6.4 ms, 7.05 with run(); matrix cores busy 67 and 54 % of the cycles.)
  template <typename F>
  __device__ __forceinline__ void run_rolling(typename Core<T>::acc_t (&acc)[S::TN][S::TM], const int count, F&& next) {
    static_assert(DIRECT && sizeof(T) == 2 && S::NB == 2 && S::TM == 8 && S::TN == 4, "");
    constexpr int STEPS = S::TM * PIECES / 4, AHEAD = 3, LAST = STEPS - 2;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wr = wave / S::WN * S::TM, wc = wave % S::WN * S::TN;
    piece_t cf[2][S::TN], rf[4];
    auto col = [&](const char* const slab, const int h, const int a) { cf[h][a] = CS::fragment(slab + 16 * PIECES * S::BM, wc + a, h); };
    auto row = [&](const char* const slab, const int i) { rf[i % 4] = RS::fragment(slab, wr + i % S::TM, i / S::TM); };
    auto products = [&](const int i) {
#pragma unroll
      for (int a = 0; a < S::TN; ++a) Core<T>::mma(cf[i / S::TM][a], rf[i % 4], acc[a][i % S::TM]);
      __builtin_amdgcn_sched_barrier(0);
    };
    // Steps from 0 to `end` - 1 of a slab.
    auto steps = [&](const char* const slab, auto end) {
#pragma unroll
      for (int i = 0; i < decltype(end)::value; ++i) {
        if (i + AHEAD < STEPS) row(slab, i + AHEAD);
        if (i >= AHEAD && i < AHEAD + S::TN) col(slab, 1, i - AHEAD);
        products(i);
      }
    };
    // What stands in front of step 0: without the third row, whose registers step 14 of the slab before still needs.
    auto head = [&](const char* const slab) {
#pragma unroll
      for (int a = 0; a < S::TN; ++a) col(slab, 0, a);
      row(slab, 0);
      row(slab, 1);
    };
    using std::integral_constant;
    typedef integral_constant<int, LAST> last;
    typedef integral_constant<int, STEPS> all;
    auto onward = [&] {
      to = to + 1 == S::NB ? 0 : to + 1;
      at = at + 1 == S::NB ? 0 : at + 1;
    };
    int left = count;
    bool headed = false;               // the first fragments of the slab to be multiplied are on their way, and the next slab is
    const int64_t end = kend - (rs.spare() > cs.spare() ? rs.spare() : cs.spare());
    const int64_t whole = rquick && cquick && k < end ? (end - k) / BK : 0;
    int steady = __builtin_amdgcn_readfirstlane(whole < left - ahead ? (int)whole : left - ahead);
    if (ahead == S::NB - 1 && steady > 0) {
      left -= steady - 1;
      headed = true;
      const char *rfrom = gemm_scalar(rs.base(k)), *cfrom = gemm_scalar(cs.base(k));
      const int64_t rstep = gemm_scalar((int64_t)(rs.base(k + BK) - rs.base(k))), cstep = gemm_scalar((int64_t)(cs.base(k + BK) - cs.base(k)));
      k += (int64_t)steady * BK;
      auto load_rows = [&] {
#pragma unroll
        for (int v = 0; v < RS::NP; ++v) rs.direct(rfrom, v, lds0 + to * S::SLAB);
        rfrom += rstep;
      };
      auto load_cols = [&] {
#pragma unroll
        for (int v = 0; v < CS::NP; ++v) cs.direct(cfrom, v, lds0 + to * S::SLAB + 16 * PIECES * S::BM);
        cfrom += cstep;
      };
      gemm_landed<0>();
      load_rows();
      load_cols();
      head(lds + at * S::SLAB);
      row(lds + at * S::SLAB, 2);
      for (; steady > 1; --steady) {
        steps(lds + at * S::SLAB, last{});
        gemm_landed<0>();              // the next slab, of all wavefronts; this one's fragments are in registers
        onward();
        head(lds + at * S::SLAB);
        __builtin_amdgcn_sched_barrier(0);
        products(LAST);
        row(lds + at * S::SLAB, 2);
        load_rows();
        __builtin_amdgcn_sched_barrier(0);
        products(LAST + 1);
        load_cols();
      }
    }
    for (; left > 0; --left) {
      const char* const slab = lds + at * S::SLAB;
      if (!headed) {
        --ahead;
        gemm_landed<0>();
        bring(next);
        head(slab);
        row(slab, 2);
      }
      steps(slab, all{});
      at = at + 1 == S::NB ? 0 : at + 1;
      if (headed) to = to + 1 == S::NB ? 0 : to + 1;
      headed = false;
    }
  }
};

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

// An operand with what is to be known of its place: offsets within a slab of B rows in 32 bits; pieces that can go straight to
// LDS, with rows on 16 bytes.
template <typename T, bool OUTER, int B>
Operand<T> gemm_operand(const void* p, const int64_t stride, const int64_t rows, const int64_t k) {
  const int64_t bytes = stride * (int64_t)sizeof(T), lines = OUTER ? k : rows;
  const bool near = bytes < (int64_t(1) << 31) / (B > 64 ? B : 64);
  const bool straight = near && (uintptr_t)p % 16 == 0 && (lines == 1 || bytes % 16 == 0);
  return Operand<T>{(const T*)p, stride, rows, near, straight};
}

// A launch holds fewer than 2^32 threads: f(first, count) for runs of workgroups that stay below that.
template <typename F>
void gemm_launches(const int64_t blocks, const int threads, F&& f) {
  const int64_t most = (int64_t)UINT32_MAX / threads;
  for (int64_t first = 0; first < blocks; first += most) f(first, dim3((unsigned)(blocks - first < most ? blocks - first : most)));
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
