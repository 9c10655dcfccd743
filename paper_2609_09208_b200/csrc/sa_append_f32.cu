// append_qkv_kernel for projections in FP32.
#include "sa_append.cuh"

namespace sa {

cudaError_t launch_append_f32(const AppendArgs& a, int d, int tokens, cudaStream_t s) { return launch_append_typed<float>(a, d, tokens, s); }

}  // namespace sa
