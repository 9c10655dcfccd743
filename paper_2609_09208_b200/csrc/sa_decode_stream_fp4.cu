// Instantiations of the decode kernel of one block per SM (see sa_decode_stream.cuh): the 4-bit cache.
#include "sa_decode_stream.cuh"

namespace sa {
template <int D>
static void launch(const DecodeArgs& a, cudaStream_t s) { a.gt <= 4 ? launch_stream<D, FMT_FP4_PAIR, 33>(a, s) : launch_stream<D, FMT_FP4, 33>(a, s); }
void launch_stream_fp4(int d, const DecodeArgs& a, cudaStream_t s) { d == 64 ? launch<64>(a, s) : launch<128>(a, s); }
}  // namespace sa
