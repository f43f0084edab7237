// gemm_to_lds with a base that comes out of vector registers and out of scalar ones, for a look at the code that comes out
// (compiled, not run).
#include "../../paper_2503_04424_amd/csrc/kernels_gemm.h"

__global__ void form(const char* const* from, float* to, int rows) {
  __shared__ __attribute__((aligned(16))) float lds[4096];
  const unsigned at = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(mdet::gemm_lds_ptr)(char*)lds);
  const char* vector = from[threadIdx.x];
  for (int r = 0; r < rows; ++r) {
    mdet::gemm_to_lds(vector, 16u * threadIdx.x, at + 1024u * (unsigned)r);
    vector += (uintptr_t)to[threadIdx.x + r];
    mdet::gemm_to_lds(vector, 16u * threadIdx.x, at + 2048u);
    mdet::gemm_to_lds(from[r], 16u * threadIdx.x, at + 4096u);
  }
  mdet::gemm_landed<0>();
  to[threadIdx.x] = lds[threadIdx.x];
}
