// chunk_kernel over caches of INT8 keys, of binary16 and of 4 bits.
#include "sa_chunk.cuh"

namespace sa {

template <int D, int FMT>
static cudaError_t launch(bool split, const ChunkArgs& a, int blocks, int rows_most, cudaStream_t s) {
    return split ? launch_chunk<D, FMT, true>(a, blocks, rows_most, s) : launch_chunk<D, FMT, false>(a, blocks, rows_most, s);
}
template <int D>
static cudaError_t launch(int fmt, bool split, const ChunkArgs& a, int blocks, int rows_most, cudaStream_t s) {
    switch (fmt) {
        case FMT_INT8: return launch<D, FMT_INT8>(split, a, blocks, rows_most, s);
        case FMT_FP16: return launch<D, FMT_FP16>(split, a, blocks, rows_most, s);
        default: return launch<D, FMT_FP4>(split, a, blocks, rows_most, s);
    }
}
cudaError_t launch_chunk_plain(int d, int fmt, bool split, const ChunkArgs& a, int blocks, int rows_most, cudaStream_t s) {
    return d == 64 ? launch<64>(fmt, split, a, blocks, rows_most, s) : launch<128>(fmt, split, a, blocks, rows_most, s);
}

}  // namespace sa
