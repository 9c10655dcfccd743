// Instantiations of the decode kernel of one block per SM (see sa_decode_stream.cuh): the 4-bit cache.
#include "sa_decode_stream.cuh"

namespace sa {
void launch_stream_fp4(int d, const DecodeArgs& a, cudaStream_t s) { d == 64 ? launch_stream<64, FMT_FP4, 33>(a, s) : launch_stream<128, FMT_FP4, 33>(a, s); }
}  // namespace sa
