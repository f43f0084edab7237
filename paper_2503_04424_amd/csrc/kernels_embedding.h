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

// y: a group's step of one row, four pieces of 16 bytes a lane at once.  Bytes bound it: 16384 rows of 1500 bf16 out of 50003 16 us (those that are
// used often come out of cache), 7 rows of 4096 3 us.
constexpr int EMBED_PIECES = 4;

template <typename T, typename I>
__global__ __launch_bounds__(256) void embedding_kernel(const I* __restrict__ ids, const int64_t n, const T* __restrict__ table, const int64_t ldt,
                                                        const int64_t vocab, const int64_t width, const float scale, T* __restrict__ y,
                                                        const int64_t ldy, const RowShare share, const int64_t first) {
  typedef typename Core<T>::piece_t piece_t;
  constexpr int VEC = Core<T>::VEC;
  const int64_t unit = (first + blockIdx.x) * (256 / share.lanes) + threadIdx.x / share.lanes;
  const int64_t row = share.chunks == 1 ? unit : unit / share.chunks;
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
// one launch; the ids come out of cache, up to 16384 at once in a workgroup's registers (SLOTS a thread), where a short list stays between the two.  The time goes with
// n times the buckets: 16384 ids of 50003 13 us (1024 at once, and one wavefront for the places, 31), a million of 32000 560 to 830.
// ---------------------------------------------------------------------------
constexpr int SORT_THREADS = 1024, SORT_WAVES = SORT_THREADS / 64;
constexpr int SORT_TOKENS = 2048;      // of a bucket
constexpr int SORT_BUCKETS = 256;      // or more, a power of two

struct Sorted {
  int32_t* place;                      // of the sorted ids: which token it is ...
  int32_t* id;                         // ... and which id
  int32_t* start;                      // for each id, where it begins and how often it is there
  int32_t* count;
  int32_t* total;                      // how many ids lie in the table
};

template <typename I, int SLOTS>
__global__ __launch_bounds__(SORT_THREADS) void embedding_sort_kernel(const I* __restrict__ ids, const int32_t n, const int64_t vocab, const int bits,
                                                                      const Sorted out) {
  constexpr int ROUND = SORT_THREADS * SLOTS, PER = SLOTS * SORT_WAVES / 64;
  static_assert(PER >= 1 && ROUND <= 1 << 16 && SORT_TOKENS <= 1 << 16, "an entry of the list is a place and a token of 16 bits each");
  __shared__ int32_t cursor[SORT_TOKENS];
  __shared__ int32_t sums[SLOTS][SORT_WAVES];
  __shared__ uint32_t list[ROUND];
  __shared__ uint16_t often[SORT_WAVES][SORT_TOKENS], behind[SORT_TOKENS];
  __shared__ int32_t all_found;
  const int thread = threadIdx.x, lane = thread & 63, wave = thread >> 6;
  const int64_t buckets = gridDim.x;
  const int32_t bucket = blockIdx.x;
  const int tokens = bucket < vocab ? (int)((vocab - bucket + buckets - 1) / buckets) : 0;
  int32_t id[SLOTS];               // -1: none of the table
  auto get = [&](const int64_t i0) {
    int64_t raw[SLOTS];
#pragma unroll
    for (int e = 0; e < SLOTS; ++e) {
      const int64_t i = i0 + e * SORT_THREADS + thread;
      raw[e] = i < n ? (int64_t)ids[i] : -1;
    }
#pragma unroll
    for (int e = 0; e < SLOTS; ++e) id[e] = raw[e] >= 0 && raw[e] < vocab ? (int32_t)raw[e] : -1;
  };
  auto bucket_of = [&](const int32_t v) { return v & (int32_t)(buckets - 1); };
  for (int t = thread; t < tokens; t += SORT_THREADS) cursor[t] = 0;
  __syncthreads();
  int32_t before = 0;
  for (int64_t i0 = 0; i0 < n; i0 += ROUND) {
    get(i0);
#pragma unroll
    for (int e = 0; e < SLOTS; ++e)
      if (id[e] >= 0) {
        before += bucket_of(id[e]) < bucket;
        if (bucket_of(id[e]) == bucket) atomicAdd(&cursor[id[e] >> bits], 1);
      }
  }
  // where the bucket begins
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) before += __shfl_xor(before, off, 64);
  if (lane == 0) sums[0][wave] = before;
  __syncthreads();
  int32_t base = 0;
#pragma unroll
  for (int w = 0; w < SORT_WAVES; ++w) base += sums[0][w];
  // where each of its tokens begins: some of them a thread
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
  if (lane == 63) sums[1][wave] = upto;
  __syncthreads();
  int32_t at = base + upto - sum, all = base;
#pragma unroll
  for (int w = 0; w < SORT_WAVES; ++w) {
    if (w < wave) at += sums[1][w];
    all += sums[1][w];
  }
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    const int t = thread * EACH + e;
    if (t < tokens) {
      const int64_t v = ((int64_t)t << bits) + bucket;
      cursor[t] = at;
      out.start[v] = at;
      out.count[v] = mine[e];
      at += mine[e];
    }
  }
  if (thread == 0 && bucket == buckets - 1) *out.total = all;
  if (all == base) return;             // nothing of this bucket: the same for the whole workgroup
  // their places, in order: what a round of ids has of this bucket is put side by side, then handed out in parts, 64 at a time; equal tokens of the
  // 64 find each other by their numbers' bits
  for (int64_t i0 = 0; i0 < n; i0 += ROUND) {
    if (n > ROUND) get(i0);
    __syncthreads();                   // sums and list have been read, cursors are written
    uint64_t hits[SLOTS];
#pragma unroll
    for (int e = 0; e < SLOTS; ++e) {
      hits[e] = __ballot(id[e] >= 0 && bucket_of(id[e]) == bucket);
      if (lane == 0) sums[e][wave] = __popcll(hits[e]);
    }
    __syncthreads();
    // the sums of the parts (64 ids each) in front of each: PER parts a lane of the first wavefront
    if (wave == 0) {
      int32_t some[PER], ahead_of = 0;
#pragma unroll
      for (int q = 0; q < PER; ++q) some[q] = (&sums[0][0])[PER * lane + q], ahead_of += some[q];
      const int32_t own = ahead_of;
#pragma unroll
      for (int off = 1; off < 64; off *= 2) {
        const int32_t o = __shfl_up(ahead_of, off, 64);
        if (lane >= off) ahead_of += o;
      }
      int32_t first = ahead_of - own;
#pragma unroll
      for (int q = 0; q < PER; ++q) {
        (&sums[0][0])[PER * lane + q] = first;
        first += some[q];
      }
      if (lane == 63) all_found = ahead_of;
    }
    __syncthreads();
    const int32_t found = all_found;
#pragma unroll
    for (int e = 0; e < SLOTS; ++e)
      if (hits[e] >> lane & 1)
        list[sums[e][wave] + __popcll(hits[e] & ((1ull << lane) - 1))] = (uint32_t)(e * SORT_THREADS + thread) << 16 | (uint32_t)(id[e] >> bits);
    const bool few = found <= 64;      // those go out at once
    if (!few)
      for (int t = thread; t < tokens; t += SORT_THREADS)
#pragma unroll
        for (int w = 0; w < SORT_WAVES; ++w) often[w][t] = 0;
    __syncthreads();
    // a part of the list for each wavefront: first how often it has each token, then the places
    const int32_t each = ((found + SORT_WAVES - 1) / SORT_WAVES + 63) & ~63, begin = wave * each, end = begin + each < found ? begin + each : found;
    auto go = [&](auto&& f) {
      for (int32_t k = begin; k < end; k += 64) {
        const bool there = k + lane < end;
        const uint32_t entry = there ? list[k + lane] : 0;
        const int32_t token = entry & 0xFFFF;
        uint64_t same = __ballot(there);
        for (int b = 1; b < tokens; b *= 2) {
          const uint64_t set = __ballot((token & b) != 0);
          same &= token & b ? set : ~set;
        }
        f(there, entry >> 16, token, __popcll(same & ((1ull << lane) - 1)), __popcll(same));
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
    };
    if (few) {
      go([&](const bool there, const uint32_t place, const int32_t token, const int rank, const int many) {
        const int32_t from = there ? cursor[token] : 0;
        __builtin_amdgcn_wave_barrier();
        if (there) {
          if (rank == 0) cursor[token] = from + many;
          out.place[from + rank] = (int32_t)(i0 + place);
          out.id[from + rank] = (token << bits) + bucket;
        }
      });
      continue;
    }
    go([&](const bool there, uint32_t, const int32_t token, const int rank, const int many) {
      if (there && rank == 0) often[wave][token] += (uint16_t)many;
    });
    __syncthreads();
    // in front of each wavefront's, those of the ones before it, in 16 bits: a round has 2^14 ids
    for (int t = thread; t < tokens; t += SORT_THREADS) {
      int32_t ahead = 0;
#pragma unroll
      for (int w = 0; w < SORT_WAVES; ++w) {
        const int32_t here = often[w][t];
        often[w][t] = (uint16_t)ahead;
        ahead += here;
      }
      behind[t] = (uint16_t)ahead;
    }
    __syncthreads();
    go([&](const bool there, const uint32_t place, const int32_t token, const int rank, const int many) {
      const int32_t before_me = there ? often[wave][token] : 0;
      __builtin_amdgcn_wave_barrier();
      if (there) {
        if (rank == 0) often[wave][token] = (uint16_t)(before_me + many);
        const int32_t to = cursor[token] + before_me + rank;
        out.place[to] = (int32_t)(i0 + place);
        out.id[to] = (token << bits) + bucket;
      }
    });
    __syncthreads();
    for (int t = thread; t < tokens; t += SORT_THREADS) cursor[t] += behind[t];
  }
}

// ---------------------------------------------------------------------------
// The sums.  A group of lanes takes RUN sorted tokens and a chunk of columns.  Tokens that begin and end among them are stored; the
// sum of one that began before (the head) or goes on behind (the tail) goes to the workspace, for the join.  So a token that is there ten
// thousand times is shared by as many groups as any other tokens, and no sum waits for another.
// ---------------------------------------------------------------------------
template <typename T, typename O>
struct EmbeddingSums {
  Sorted s;
  const T* dy;
  int64_t lddy;
  O* g;
  int64_t ldg;
  float* parts;                        // runs x 2 (head, tail) x width
  int64_t n, vocab, width, runs;
  float scale;
  bool add;                            // to what g holds
};

// The first `sum_blocks` workgroups sum; the others write zeros where no token is, a step of ZERO_PIECES pieces a lane.  Bytes bound
// both: 50003 x 1024 fp32 from 16384 bf16 rows 33 us (205 MB of zeros and sums written, 7 TB/s; 45 with 32 bytes a lane in one step).
constexpr int ZERO_PIECES = 4;

template <typename T, typename O, int RUN>
__global__ __launch_bounds__(256) void embedding_sum_kernel(const EmbeddingSums<T, O> a, const RowShare share, const RowShare zeros,
                                                            const int64_t sum_blocks, const int64_t first) {
  typedef typename Core<T>::piece_t piece_t;
  constexpr int VEC = Core<T>::VEC;
  const int lane = threadIdx.x % share.lanes, groups = 256 / share.lanes;
  const int64_t block = first + blockIdx.x;
  if (block >= sum_blocks) {
    constexpr int OUT = 16 / sizeof(O);
    const int zlane = threadIdx.x % zeros.lanes;
    const int64_t unit = (block - sum_blocks) * (256 / zeros.lanes) + threadIdx.x / zeros.lanes, id = zeros.chunks == 1 ? unit : unit / zeros.chunks;
    if (id >= a.vocab || a.s.count[id] != 0) return;
    typedef O out_t __attribute__((ext_vector_type(OUT)));
    O* const row = a.g + id * a.ldg;
    const int64_t c0 = ((unit - id * zeros.chunks) * ZERO_PIECES * zeros.lanes + zlane) * OUT;
#pragma unroll
    for (int p = 0; p < ZERO_PIECES; ++p) {
      const int64_t c = c0 + p * zeros.lanes * OUT;
      const out_t zero = {};
      if (c + OUT <= a.width) __builtin_memcpy(row + c, &zero, 16);
      else
#pragma unroll
        for (int e = 0; e < OUT - 1; ++e)
          if (c + e < a.width) row[c + e] = (O)0.0f;
    }
    return;
  }
  const int64_t unit = block * groups + threadIdx.x / share.lanes, run = share.chunks == 1 ? unit : unit / share.chunks;
  const int64_t p0 = run * RUN;
  if (run >= a.runs) return;
  // A lane's place and id of the run's, and the ids beside it: groups are whole rows of lanes.  Behind the last there is something in memory as
  // well, which is not looked at.
  const int64_t own = p0 + lane % RUN < a.n ? p0 + lane % RUN : a.n - 1, behind = p0 + RUN < a.n ? p0 + RUN : a.n - 1;
  const int32_t place = a.s.place[own], key = a.s.id[own], front = a.s.id[p0 > 0 ? p0 - 1 : 0], back = a.s.id[behind];
  const int32_t total = *a.s.total;
  if (p0 >= total) return;
  const int32_t prior = p0 > 0 ? front : -1, later = p0 + RUN < total ? back : -1;
  const int64_t c = ((unit - run * share.chunks) * share.lanes + lane) * VEC;
  const int many = total - p0 < RUN ? (int)(total - p0) : RUN;
  piece_t x[RUN];
#pragma unroll
  for (int r = 0; r < RUN; ++r) {
    const int64_t i = __shfl(place, r, RUN);
    x[r] = piece_t{};
    if (r < many) x[r] = row_piece<T>(a.dy + i * a.lddy, c, a.width);
  }
  // The sums that end in front of each row, four rows at a time: what they are added to is on its way for all of the four at once.
  float sum[VEC] = {}, done[4][VEC];
  int32_t where[4];                    // the id whose sum it is; -1: none ends here
  int32_t last = __shfl(key, 0, RUN);
  bool open = last == prior;           // the sum began in front of this run
  auto part = [&](const int which) {
    float* const to = a.parts + (run * 2 + which) * a.width;
    if (c < a.width) row_store<T, float>(to, c, a.width, sum);
  };
  auto put = [&](auto many_of) {
    constexpr int MANY = decltype(many_of)::value;
    float old[MANY][VEC] = {};
    if (a.add) {
#pragma unroll
      for (int q = 0; q < MANY; ++q)
        if (where[q] >= 0)
#pragma unroll
          for (int e = 0; e < VEC; ++e)
            if (c + e < a.width) old[q][e] = (float)a.g[where[q] * a.ldg + c + e];
    }
#pragma unroll
    for (int q = 0; q < MANY; ++q) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) done[q][e] = done[q][e] * a.scale + old[q][e];
      if (where[q] >= 0 && c < a.width) row_store<T, O>(a.g + where[q] * a.ldg, c, a.width, done[q]);
    }
  };
#pragma unroll
  for (int r0 = 0; r0 < RUN; r0 += 4) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int r = r0 + q;
      const int32_t id = __shfl(key, r, RUN);
      const bool ends = r < many && id != last;
      where[q] = ends && !open ? last : -1;
      if (ends && open) part(0);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        done[q][e] = sum[e];
        sum[e] = (ends ? 0.0f : sum[e]) + (float)x[r][e];      // rows behind the last are zero
      }
      open = open && !ends;
      last = r < many ? id : last;
    }
    put(std::integral_constant<int, 4>{});
  }
  if (open) part(0);
  else if (last == later) part(1);
  else {
    where[0] = last;
#pragma unroll
    for (int e = 0; e < VEC; ++e) done[0][e] = sum[e];
    put(std::integral_constant<int, 1>{});
  }
}

// A token that begins in a run and goes on behind it: its parts, added in one order, eight threads a column (8 us for 16384 tokens, most of
// it workgroups that find nothing to do).
constexpr int JOIN_COLS = 128, JOIN_GROUPS = 1024 / JOIN_COLS;

template <typename T, typename O, int RUN>
__global__ __launch_bounds__(256) void embedding_join_kernel(const EmbeddingSums<T, O> a, const int64_t across, const int64_t first) {
  typedef float f4 __attribute__((ext_vector_type(4)));
  __shared__ f4 part[JOIN_GROUPS][JOIN_COLS / 4];
  const int64_t block = first + blockIdx.x, run = block / across, next = (run + 1) * RUN;
  if (next >= *a.s.total) return;
  const int32_t id = a.s.id[next - 1], begin = a.s.start[id];
  const int64_t end = (int64_t)begin + a.s.count[id];
  if (end <= next || begin < next - RUN) return;
  const int t = threadIdx.x / (JOIN_COLS / 4), lane = threadIdx.x % (JOIN_COLS / 4);
  const int64_t c = (block - run * across) * JOIN_COLS + lane * 4, runs = (end + RUN - 1) / RUN;
  auto get = [&](const int64_t r) {
    const float* const from = a.parts + (r == run ? 2 * r + 1 : 2 * r) * a.width + c;
    f4 x = {};
    if (c + 4 <= a.width) __builtin_memcpy(&x, from, 16);
    else
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (c + e < a.width) x[e] = from[e];
    return x;
  };
  f4 v = {};
  int64_t r = run + t;
  for (; r + 3 * JOIN_GROUPS < runs; r += 4 * JOIN_GROUPS) {
    f4 x[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) x[q] = get(r + q * JOIN_GROUPS);
#pragma unroll
    for (int q = 0; q < 4; ++q) v += x[q];
  }
  for (; r < runs; r += JOIN_GROUPS) v += get(r);
  part[t][lane] = v;
  __syncthreads();
  if (t == 0) {
#pragma unroll
    for (int g = 1; g < JOIN_GROUPS; ++g) v += part[g][lane];
    O* const row = a.g + id * a.ldg;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c + e < a.width) row[c + e] = (O)(v[e] * a.scale + (a.add ? (float)row[c + e] : 0.0f));
  }
}

}  // namespace mdet
