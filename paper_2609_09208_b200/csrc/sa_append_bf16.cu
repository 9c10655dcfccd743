// append_qkv_kernel for projections in bfloat16.
#include "sa_append.cuh"

namespace sa {

cudaError_t launch_append_bf16(const AppendArgs& a, int d, int tokens, cudaStream_t s) { return launch_append_typed<__nv_bfloat16>(a, d, tokens, s); }

}  // namespace sa
