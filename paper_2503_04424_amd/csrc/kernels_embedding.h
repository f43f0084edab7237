// Rows of a table by token numbers, and the gradient of the table.
//
//   y_i = scale table[id_i];  G_v = scale (sum over i with id_i = v of dy_i)
//
// An id outside of the table gives a row of zeros and has no part in the gradient.  The gradient's tokens are sorted first, by
// their number and, within one, by their place, so that every sum has one order; sums are fp32, rounded once.
#pragma once
#include "kernels_rows.h"

namespace mdet {

// How a row is shared out: groups of `lanes` neighbouring lanes (16, 32 or 64), PIECES pieces of 16 bytes each a step, `chunks`
// steps a row.
struct RowShare {
  int lanes;
  int64_t chunks;
};

// y: a group's step of one row.  Bytes bound it.
constexpr int EMBED_PIECES = 4;

template <typename T, typename I>
__global__ __launch_bounds__(256) void embedding_kernel(const I* __restrict__ ids, const int64_t n, const T* __restrict__ table, const int64_t ldt,
                                                        const int64_t vocab, const int64_t width, const float scale, T* __restrict__ y,
                                                        const int64_t ldy, const RowShare share, const int64_t first) {
  typedef typename Core<T>::piece_t piece_t;
  constexpr int VEC = Core<T>::VEC;
  const int64_t unit = (first + blockIdx.x) * (256 / share.lanes) + threadIdx.x / share.lanes;
  const int64_t row = unit / share.chunks;
  if (row >= n) return;
  const int64_t c0 = (unit - row * share.chunks) * share.lanes * EMBED_PIECES * VEC + threadIdx.x % share.lanes * VEC;
  const int64_t step = (int64_t)share.lanes * VEC, id = (int64_t)ids[row];
  T* const to = y + row * ldy;
  piece_t x[EMBED_PIECES] = {};
  if (id >= 0 && id < vocab) {
    const T* const from = table + id * ldt;
#pragma unroll
    for (int p = 0; p < EMBED_PIECES; ++p) x[p] = row_piece<T>(from, c0 + p * step, width);
  }
#pragma unroll
  for (int p = 0; p < EMBED_PIECES; ++p) {
    float v[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = (id >= 0 && id < vocab) ? (float)x[p][e] * scale : 0.0f;
    if (c0 + p * step < width) row_store<T, T>(to, c0 + p * step, width, v);
  }
}

// ---------------------------------------------------------------------------
// The sort.  Token v belongs to bucket v % buckets (so that the frequent ones, which have small numbers as a rule, lie in
// different ones), and a workgroup to each bucket, which goes through all of the ids twice: to count its own, token by token, and
// those of the buckets in front of it; then to write their places down, in order.  That needs no word between workgroups and
// one launch; the ids come out of cache.
// ---------------------------------------------------------------------------
constexpr int SORT_THREADS = 1024, SORT_WAVES = SORT_THREADS / 64;
constexpr int SORT_TOKENS = 4096;      // of a bucket
constexpr int SORT_BUCKETS = 256;      // or more, a power of two

struct Sorted {
  int32_t* place;                      // of the sorted ids: which token it is ...
  int32_t* id;                         // ... and which id
  int32_t* start;                      // for each id, where it begins and how often it is there
  int32_t* count;
  int32_t* total;                      // how many ids lie in the table
};

template <typename I>
__global__ __launch_bounds__(SORT_THREADS) void embedding_sort_kernel(const I* __restrict__ ids, const int32_t n, const int64_t vocab, const int bits,
                                                                      const Sorted out) {
  __shared__ int32_t cursor[SORT_TOKENS];
  __shared__ int32_t wave_sum[SORT_WAVES];
  __shared__ int32_t list_place[SORT_THREADS], list_token[SORT_THREADS];
  const int thread = threadIdx.x, lane = thread & 63, wave = thread >> 6;
  const int64_t bucket = blockIdx.x, buckets = gridDim.x;
  const int tokens = bucket < vocab ? (int)((vocab - bucket + buckets - 1) / buckets) : 0;
  for (int t = thread; t < tokens; t += SORT_THREADS) cursor[t] = 0;
  __syncthreads();
  int32_t before = 0;
  for (int32_t i = thread; i < n; i += SORT_THREADS) {
    const int64_t id = (int64_t)ids[i];
    if (id < 0 || id >= vocab) continue;
    const int64_t b = id & (buckets - 1);
    before += b < bucket;
    if (b == bucket) atomicAdd(&cursor[id >> bits], 1);
  }
  // where the bucket begins
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) before += __shfl_xor(before, off, 64);
  if (lane == 0) wave_sum[wave] = before;
  __syncthreads();
  int32_t base = 0;
#pragma unroll
  for (int w = 0; w < SORT_WAVES; ++w) base += wave_sum[w];
  // where each of its tokens begins: four of them a thread
  constexpr int EACH = SORT_TOKENS / SORT_THREADS;
  int32_t mine[EACH], sum = 0;
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    const int t = thread * EACH + e;
    mine[e] = t < tokens ? cursor[t] : 0;
    sum += mine[e];
  }
  int32_t upto = sum;
#pragma unroll
  for (int off = 1; off < 64; off *= 2) {
    const int32_t o = __shfl_up(upto, off, 64);
    if (lane >= off) upto += o;
  }
  __syncthreads();                     // wave_sum has been read
  if (lane == 63) wave_sum[wave] = upto;
  __syncthreads();
  int32_t at = base + upto - sum, all = base;
#pragma unroll
  for (int w = 0; w < SORT_WAVES; ++w) {
    if (w < wave) at += wave_sum[w];
    all += wave_sum[w];
  }
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    const int t = thread * EACH + e;
    if (t < tokens) {
      const int64_t id = ((int64_t)t << bits) + bucket;
      cursor[t] = at;
      out.start[id] = at;
      out.count[id] = mine[e];
      at += mine[e];
    }
  }
  if (thread == 0 && bucket == buckets - 1) *out.total = all;
  if (all == base) return;             // nothing of this bucket: the same for the whole workgroup
  __syncthreads();
  // their places, in order: what a round of ids has of this bucket is put side by side, then handed out by one wavefront after
  // the other, 64 at a time; equal tokens of the 64 find each other by their numbers' bits
  for (int64_t i0 = 0; i0 < n; i0 += SORT_THREADS) {
    const int64_t i = i0 + thread, id = i < n ? (int64_t)ids[i] : -1;
    const bool hit = id >= 0 && id < vocab && (id & (buckets - 1)) == bucket;
    const uint64_t hits = __ballot(hit);
    if (lane == 0) wave_sum[wave] = __popcll(hits);
    __syncthreads();
    int32_t where = __popcll(hits & ((1ull << lane) - 1)), found = 0;
#pragma unroll
    for (int w = 0; w < SORT_WAVES; ++w) {
      if (w < wave) where += wave_sum[w];
      found += wave_sum[w];
    }
    if (hit) {
      list_place[where] = (int32_t)i;
      list_token[where] = (int32_t)(id >> bits);
    }
    __syncthreads();
    if (wave == 0)
      for (int32_t k = 0; k < found; k += 64) {
        const bool there = k + lane < found;
        const int32_t token = there ? list_token[k + lane] : 0;
        uint64_t same = __ballot(there);
        for (int b = 1; b < tokens; b *= 2) {
          const uint64_t set = __ballot((token & b) != 0);
          same &= token & b ? set : ~set;
        }
        const int rank = __popcll(same & ((1ull << lane) - 1));
        const int32_t from = there ? cursor[token] : 0;
        __builtin_amdgcn_wave_barrier();
        if (there) {
          if (rank == 0) cursor[token] = from + __popcll(same);
          out.place[from + rank] = list_place[k + lane];
          out.id[from + rank] = (int32_t)((token << bits) + (int32_t)bucket);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
    // the next round writes the list behind its first barrier, which wavefront 0 reaches when it is through with this one
  }
}

// ---------------------------------------------------------------------------
// The sums.  A group of lanes takes RUN sorted tokens and a chunk of columns.  Tokens that begin and end among them are stored; the
// sum of one that began before (the head) or goes on behind (the tail) goes to the workspace, for the join.
// ---------------------------------------------------------------------------
constexpr int RUN = 16;

template <typename T, typename O>
struct EmbeddingSums {
  Sorted s;
  const T* dy;
  int64_t lddy;
  O* g;
  int64_t ldg;
  float* parts;                        // runs x 2 (head, tail) x width
  int64_t vocab, width, runs;
  float scale;
  bool add;                            // to what g holds
};

template <typename T, typename O>
__device__ __forceinline__ void embedding_put(const EmbeddingSums<T, O>& a, const int64_t id, const int64_t c, float (&v)[Core<T>::VEC]) {
  constexpr int VEC = Core<T>::VEC;
  O* const row = a.g + id * a.ldg;
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    v[e] *= a.scale;
    if (a.add && c + e < a.width) v[e] += (float)row[c + e];
  }
  row_store<T, O>(row, c, a.width, v);
}

// The first `sum_blocks` workgroups sum; the others write zeros where no token is.
template <typename T, typename O>
__global__ __launch_bounds__(256) void embedding_sum_kernel(const EmbeddingSums<T, O> a, const RowShare share, const int64_t sum_blocks,
                                                            const int64_t first) {
  typedef typename Core<T>::piece_t piece_t;
  constexpr int VEC = Core<T>::VEC;
  const int lane = threadIdx.x % share.lanes, groups = 256 / share.lanes;
  const int64_t block = first + blockIdx.x;
  if (block >= sum_blocks) {
    const int64_t unit = (block - sum_blocks) * groups + threadIdx.x / share.lanes, id = unit / share.chunks;
    if (id >= a.vocab || a.s.count[id] != 0) return;
    const int64_t c = ((unit - id * share.chunks) * share.lanes + lane) * VEC;
    const float zero[VEC] = {};
    if (c < a.width) row_store<T, O>(a.g + id * a.ldg, c, a.width, zero);
    return;
  }
  const int64_t unit = block * groups + threadIdx.x / share.lanes, run = unit / share.chunks;
  const int32_t total = *a.s.total;
  const int64_t p0 = run * RUN;
  if (p0 >= total) return;
  const int64_t c = ((unit - run * share.chunks) * share.lanes + lane) * VEC;
  const int many = total - p0 < RUN ? (int)(total - p0) : RUN;
  // a lane's place and id of the sixteen: groups are whole rows of sixteen lanes
  const int mine = lane % RUN < many ? lane % RUN : many - 1;
  const int32_t place = a.s.place[p0 + mine], key = a.s.id[p0 + mine];
  const int32_t prior = p0 > 0 ? a.s.id[p0 - 1] : -1, later = p0 + many < total ? a.s.id[p0 + many] : -1;
  piece_t x[RUN];
#pragma unroll
  for (int r = 0; r < RUN; ++r) {
    const int64_t i = __shfl(place, r, RUN);
    x[r] = piece_t{};
    if (r < many) x[r] = row_piece<T>(a.dy + i * a.lddy, c, a.width);
  }
  float sum[VEC] = {};
  bool open = false;                   // the sum began in front of this run
  int32_t last = prior;
  auto part = [&](const int which) {
    float* const to = a.parts + (run * 2 + which) * a.width;
    if (c < a.width) row_store<T, float>(to, c, a.width, sum);
  };
#pragma unroll
  for (int r = 0; r < RUN; ++r) {
    const int32_t id = __shfl(key, r, RUN);
    if (r < many) {
      if (r == 0) open = id == prior;
      else if (id != last) {
        if (open) part(0);
        else if (c < a.width) embedding_put(a, last, c, sum);
        open = false;
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[e] = 0.0f;
      }
      last = id;
#pragma unroll
      for (int e = 0; e < VEC; ++e) sum[e] += (float)x[r][e];
    }
  }
  if (open) part(0);
  else if (last == later) part(1);
  else if (c < a.width) embedding_put(a, last, c, sum);
}

// A token that begins in run `blockIdx / chunks` and goes on behind it: its parts, added in one order, sixteen threads a column.
constexpr int JOIN_COLS = 64;

template <typename T, typename O>
__global__ __launch_bounds__(256) void embedding_join_kernel(const EmbeddingSums<T, O> a, const int64_t across, const int64_t first) {
  typedef float f4 __attribute__((ext_vector_type(4)));
  __shared__ f4 part[16][JOIN_COLS / 4];
  const int64_t block = first + blockIdx.x, run = block / across, next = (run + 1) * RUN;
  if (next >= *a.s.total) return;
  const int32_t id = a.s.id[next - 1], begin = a.s.start[id];
  const int64_t end = (int64_t)begin + a.s.count[id];
  if (end <= next || begin < next - RUN) return;
  const int t = threadIdx.x / 16;
  const int64_t c = (block - run * across) * JOIN_COLS + threadIdx.x % 16 * 4;
  f4 v = {};
  for (int64_t r = run + t; r * RUN < end; r += 16) {
    const float* const from = a.parts + (r == run ? 2 * r + 1 : 2 * r) * a.width + c;
    if (c + 4 <= a.width) {
      f4 x;
      __builtin_memcpy(&x, from, 16);
      v += x;
    } else
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (c + e < a.width) v[e] += from[e];
  }
  part[t][threadIdx.x % 16] = v;
  __syncthreads();
  if (t == 0) {
#pragma unroll
    for (int r = 1; r < 16; ++r) v += part[r][threadIdx.x];
    O* const row = a.g + (int64_t)id * a.ldg;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c + e < a.width) row[c + e] = (O)(v[e] * a.scale + (a.add ? (float)row[c + e] : 0.0f));
  }
}

}  // namespace mdet
