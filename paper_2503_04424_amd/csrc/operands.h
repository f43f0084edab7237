// What the operators' entry points check of their operands: host code.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/memdet.h"

namespace mdet {

inline uint64_t up256(uint64_t x) { return (x + 255) / 256 * 256; }
inline int64_t size_of(int32_t t) { return t == MDET_F32 ? 4 : 2; }
inline bool is_type(int32_t t) { return t == MDET_F32 || t == MDET_F16 || t == MDET_BF16; }
inline int launch_status() { return hipGetLastError() == hipSuccess ? MDET_OK : MDET_EHIP; }

// Sizes whose products and byte counts stay within 64 bits.
constexpr int64_t MOST = int64_t(1) << 40;
inline bool sizes_fit(int64_t m, int64_t n, int64_t k) {
  if (m < 0 || n < 0 || k < 0 || m > MOST || n > MOST || k > MOST) return false;
  const int64_t most = int64_t(1) << 52;
  return (!n || m <= most / n) && (!k || m <= most / k) && (!k || n <= most / k);
}

// A matrix of r rows and c columns in memory: null only where it has no elements, rows that do not overlap.
inline bool matrix_ok(const void* p, int64_t r, int64_t c, int64_t ld, int64_t size) {
  if (r == 0 || c == 0) return true;
  return p && (uintptr_t)p % size == 0 && (r == 1 || ld >= c) && ld >= 0 && ld <= MOST;
}

// n consecutive elements.
inline bool vector_ok(const void* p, int64_t n, int64_t size) { return n == 0 || (p && (uintptr_t)p % size == 0); }

// Of a workspace: MDET_OK, or the error of a call that gets it.
inline int workspace_ok(const void* workspace, uint64_t bytes, uint64_t need) {
  if (need && (!workspace || (uintptr_t)workspace % 256)) return MDET_EINVAL;
  return bytes < need ? MDET_ENOMEM_DEVICE : MDET_OK;
}

}  // namespace mdet
