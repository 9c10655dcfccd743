// Instantiations of the decode kernel (see sa_decode_mma.cuh): the 4-bit cache.
#include "sa_decode_mma.cuh"

namespace sa {
template <int D>
static void launch(const DecodeArgs& a, dim3 grid, cudaStream_t s) {
    constexpr KernelShape sh = fp4_shape(D);
    if (a.gt <= 4) launch_mma<D, FMT_FP4_PAIR, 33, sh.warps, sh.blocks_per_sm, sh.stages>(a, grid, s);
    else launch_mma<D, FMT_FP4, 33, sh.warps, sh.blocks_per_sm, sh.stages>(a, grid, s);
}
void launch_mma_fp4(int d, const DecodeArgs& a, dim3 grid, cudaStream_t s) {
    if (d == 64) launch<64>(a, grid, s);
    else launch<128>(a, grid, s);
}
}  // namespace sa
