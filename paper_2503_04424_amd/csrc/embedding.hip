// C ABI of the embedding and its gradient: argument checks, workspace layout and kernel launches.  A call only queues work on
// the caller's stream; nothing is allocated and nothing is waited for.
#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>

#include "kernels_embedding.h"
#include "linear_cut.h"
#include "operands.h"

namespace {

using namespace mdet;

// Lanes for a row of this many pieces, `each` pieces a lane and step.
RowShare share_of(int64_t width, int64_t size, int each) {
  const int64_t pieces = ceil_div(width * size, 16);
  RowShare s;
  s.lanes = pieces <= 16 * each ? 16 : pieces <= 32 * each ? 32 : 64;
  s.chunks = ceil_div(pieces, (int64_t)s.lanes * each);
  return s;
}

// Ids and tokens are counted in 32 bits.
bool embedding_fits(int64_t n, int64_t vocab, int64_t width) {
  return sizes_fit(n, vocab, width) && n < INT32_MAX - 1024 && vocab <= INT32_MAX;
}
bool is_index(int32_t bits) { return bits == 32 || bits == 64; }

// Sorted tokens of a group of lanes: few while there are few groups, each of which waits for one load behind the other; more of them where the sums
// that cross runs count.  us with 4, 8 and 16: 173 tokens, rows of 40 15.3, 17.1, 21; 4096, 512 22, 25, 33 (added); 4096, 2000 40, 39, 42; 8192,
// 512 28.1, 27.5, 33; 65536, 128 75, 67, 66; 16384, 1024 of 50003 68, 59, 54; 65536, 1024 169, 137, 130.
int run_of(int64_t n, int64_t width) {
  const int64_t elements = n * width;
  return elements >= (int64_t(1) << 23) ? 16 : n < 6144 && elements < (int64_t(1) << 22) ? 4 : 8;
}

// Workspace of the gradient: the sorted ids and their places, where each id begins and how often it is there, how many there are,
// then the parts of the sums that cross runs.
struct SortLayout {
  int64_t runs;
  uint64_t id, start, count, total, parts, bytes;
};
SortLayout sort_layout(int64_t n, int64_t vocab, int64_t width) {
  SortLayout l;
  l.runs = ceil_div(n, run_of(n, width));
  l.id = up256((uint64_t)n * 4);
  l.start = l.id + up256((uint64_t)n * 4);
  l.count = l.start + up256((uint64_t)vocab * 4);
  l.total = l.count + up256((uint64_t)vocab * 4);
  l.parts = l.total + 256;
  l.bytes = l.parts + (l.runs > 1 ? up256((uint64_t)l.runs * 2 * width * 4) : 0);
  return l;
}

template <typename T, typename O, typename I>
int backward(int64_t n, const I* ids, const EmbeddingSums<T, O>& a, hipStream_t st) {
  int bits = 0;
  while ((int64_t(1) << bits) < SORT_BUCKETS || (a.vocab >> bits) >= SORT_TOKENS) ++bits;
  // ids in a thread's registers: no more than there are (sixteen and what is taken here, us of the whole call: 173 ids 15.3 and 13.8, 4096 of 512 22.0
  // and 20.2, 8192 27.3 and 26.0)
  auto sort = [&](auto slots) {
    hipLaunchKernelGGL((embedding_sort_kernel<I, decltype(slots)::value>), dim3(1u << bits), dim3(SORT_THREADS), 0, st, ids, (int32_t)n, a.vocab, bits, a.s);
  };
  if (n <= 4096) sort(std::integral_constant<int, 4>{});
  else if (n <= 8192) sort(std::integral_constant<int, 8>{});
  else sort(std::integral_constant<int, 16>{});
  const RowShare share = share_of(a.width, sizeof(T), 1);
  const int groups = 256 / share.lanes;
  const RowShare zeros = share_of(a.width, sizeof(O), ZERO_PIECES);
  const int64_t sums = ceil_div(a.runs * share.chunks, groups), empty = a.add ? 0 : ceil_div(a.vocab * zeros.chunks, 256 / zeros.lanes);
  auto go = [&](auto run) {
    constexpr int RUN = decltype(run)::value;
    gemm_launches(sums + empty, 256, [&](const int64_t first, const dim3 grid) {
      hipLaunchKernelGGL((embedding_sum_kernel<T, O, RUN>), grid, dim3(256), 0, st, a, share, zeros, sums, first);
    });
    if (a.runs <= 1) return;
    const int64_t across = ceil_div(a.width, JOIN_COLS);
    gemm_launches((a.runs - 1) * across, 256, [&](const int64_t first, const dim3 grid) {
      hipLaunchKernelGGL((embedding_join_kernel<T, O, RUN>), grid, dim3(256), 0, st, a, across, first);
    });
  };
  const int run = run_of(n, a.width);
  if (run == 4) go(std::integral_constant<int, 4>{});
  else if (run == 8) go(std::integral_constant<int, 8>{});
  else go(std::integral_constant<int, 16>{});
  return launch_status();
}

}  // namespace

extern "C" {

int mdet_embedding_workspace_query(int64_t n, int64_t vocab, int64_t width, uint64_t* bytes) {
  if (!bytes || !embedding_fits(n, vocab, width)) return MDET_EINVAL;
  *bytes = sort_layout(n, vocab, width).bytes;
  return MDET_OK;
}

int mdet_embedding_forward(int32_t dtype, int32_t index_bits, int64_t n, int64_t vocab, int64_t width, const void* ids, const void* table,
                           int64_t ldt, double scale, void* y, int64_t ldy, void* stream) {
  if (!is_type(dtype) || !is_index(index_bits) || !embedding_fits(n, vocab, width) || !std::isfinite((float)scale)) return MDET_EINVAL;
  const int64_t s = size_of(dtype);
  if (!matrix_ok(table, vocab, width, ldt, s) || !matrix_ok(y, n, width, ldy, s) || !vector_ok(ids, n, index_bits / 8)) return MDET_EINVAL;
  if (n == 0 || width == 0) return MDET_OK;
  auto call = [&](auto zero, auto index) {
    typedef decltype(zero) T;
    typedef decltype(index) I;
    const RowShare share = share_of(width, sizeof(T), EMBED_PIECES);
    gemm_launches(ceil_div(n * share.chunks, 256 / share.lanes), 256, [&](const int64_t first, const dim3 grid) {
      hipLaunchKernelGGL((embedding_kernel<T, I>), grid, dim3(256), 0, (hipStream_t)stream, (const I*)ids, n, (const T*)table, ldt, vocab, width,
                         (float)scale, (T*)y, ldy, share, first);
    });
    return launch_status();
  };
  auto typed = [&](auto index) {
    return dtype == MDET_F32 ? call(0.0f, index) : dtype == MDET_BF16 ? call((__bf16)0.0f, index) : call((_Float16)0.0f, index);
  };
  return index_bits == 32 ? typed(int32_t(0)) : typed(int64_t(0));
}

int mdet_embedding_backward(int32_t dtype, int32_t grad_dtype, int32_t index_bits, int64_t n, int64_t vocab, int64_t width, const void* ids,
                            const void* dy, int64_t lddy, double scale, int32_t accumulate, void* dtable, int64_t ldt, void* workspace,
                            uint64_t workspace_bytes, void* stream) {
  if (!is_type(dtype) || (grad_dtype != dtype && grad_dtype != MDET_F32) || !is_index(index_bits)) return MDET_EINVAL;
  if (!embedding_fits(n, vocab, width) || !std::isfinite((float)scale)) return MDET_EINVAL;
  if (!matrix_ok(dy, n, width, lddy, size_of(dtype)) || !matrix_ok(dtable, vocab, width, ldt, size_of(grad_dtype))) return MDET_EINVAL;
  if (!vector_ok(ids, n, index_bits / 8)) return MDET_EINVAL;
  const SortLayout l = sort_layout(n, vocab, width);
  const int ok = workspace_ok(workspace, workspace_bytes, l.bytes);
  if (ok != MDET_OK) return ok;
  if (vocab == 0 || width == 0 || (n == 0 && accumulate)) return MDET_OK;
  char* const ws = (char*)workspace;
  auto call = [&](auto zero, auto out, auto index) {
    typedef decltype(zero) T;
    typedef decltype(out) O;
    typedef decltype(index) I;
    const EmbeddingSums<T, O> a{{(int32_t*)ws, (int32_t*)(ws + l.id), (int32_t*)(ws + l.start), (int32_t*)(ws + l.count), (int32_t*)(ws + l.total)},
                                (const T*)dy, lddy, (O*)dtable, ldt, (float*)(ws + l.parts), n, vocab, width, l.runs, (float)scale, accumulate != 0};
    return backward<T, O, I>(n, (const I*)ids, a, (hipStream_t)stream);
  };
  auto typed = [&](auto index) {
    if (dtype == MDET_F32) return call(0.0f, 0.0f, index);
    if (dtype == MDET_BF16) return grad_dtype == MDET_F32 ? call((__bf16)0.0f, 0.0f, index) : call((__bf16)0.0f, (__bf16)0.0f, index);
    return grad_dtype == MDET_F32 ? call((_Float16)0.0f, 0.0f, index) : call((_Float16)0.0f, (_Float16)0.0f, index);
  };
  return index_bits == 32 ? typed(int32_t(0)) : typed(int64_t(0));
}

}  // extern "C"
