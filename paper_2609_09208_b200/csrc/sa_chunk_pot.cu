// chunk_kernel over caches of the power-of-two codes.
#include "sa_chunk.cuh"

namespace sa {

template <int D, int FMT>
static cudaError_t launch(bool split, const ChunkArgs& a, int blocks, int rows_most, cudaStream_t s) {
    return split ? launch_chunk<D, FMT, true>(a, blocks, rows_most, s) : launch_chunk<D, FMT, false>(a, blocks, rows_most, s);
}
template <int D>
static cudaError_t launch(int fmt, bool split, const ChunkArgs& a, int blocks, int rows_most, cudaStream_t s) {
    switch (fmt) {
        case FMT_BYTE: return launch<D, FMT_BYTE>(split, a, blocks, rows_most, s);
        case FMT_NIBBLE: return launch<D, FMT_NIBBLE>(split, a, blocks, rows_most, s);
        case FMT_PLANAR1: return launch<D, FMT_PLANAR1>(split, a, blocks, rows_most, s);
        default: return launch<D, FMT_PLANAR2>(split, a, blocks, rows_most, s);
    }
}
cudaError_t launch_chunk_pot(int d, int fmt, bool split, const ChunkArgs& a, int blocks, int rows_most, cudaStream_t s) {
    return d == 64 ? launch<64>(fmt, split, a, blocks, rows_most, s) : launch<128>(fmt, split, a, blocks, rows_most, s);
}
cudaError_t launch_chunk_lost(bool split, const ChunkArgs& a, int blocks, int rows_most, cudaStream_t s) {
    return split ? launch_chunk<64, FMT_BYTE, true, true>(a, blocks, rows_most, s) : launch_chunk<64, FMT_BYTE, false, true>(a, blocks, rows_most, s);
}

}  // namespace sa
