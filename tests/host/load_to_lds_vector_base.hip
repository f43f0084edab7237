// load_to_lds with a base that comes out of vector registers and out of scalar ones, for a look at the code that comes out
// (compiled, not run).
#include "../../paper_2503_04424_amd/csrc/kernels_update.h"

template <int SIZE, int SCOPE>
__global__ void form(const char* const* from, float* to, int rows) {
  __shared__ __attribute__((aligned(16))) float lds[4096];
  const unsigned at = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(mdet::upd_lds_ptr)lds);
  const char* vector = from[threadIdx.x];
  for (int r = 0; r < rows; ++r) {
    mdet::load_to_lds<SIZE, SCOPE>(vector, (unsigned)(SIZE * threadIdx.x), at + 1024u * (unsigned)r);
    vector += (uintptr_t)to[threadIdx.x + r];
    mdet::load_to_lds<SIZE, SCOPE>(vector, (unsigned)(SIZE * threadIdx.x), at + 2048u);
    mdet::load_to_lds<SIZE, SCOPE>(from[r], (unsigned)(SIZE * threadIdx.x), at + 4096u);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  to[threadIdx.x] = lds[threadIdx.x];
}
template __global__ void form<16, 0>(const char* const*, float*, int);
template __global__ void form<16, mdet::DEVICE_SCOPE>(const char* const*, float*, int);
template __global__ void form<4, 0>(const char* const*, float*, int);
template __global__ void form<4, mdet::DEVICE_SCOPE>(const char* const*, float*, int);
