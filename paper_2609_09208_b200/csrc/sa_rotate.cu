// sa_rotate_qkv: from a layer's projections to the rows that the cache and the decode calls take.
//
// One pass over the data: y = x / sqrt(mean(x^2) + eps) * w for every query and key head, then the rotation of its first R channels by
// the token's positions, FP32 throughout, one rounding to binary16; values are converted.  Bound by memory (each input read, each
// output written once); single tokens by latency.
//
// d / (2 P) lanes share a head vector; a lane holds two pieces of P channels whose pairs lie in the lane: pairing halves, channels
// u .. u + P - 1 and their partners; pairing neighbours, any two.  So the rotation needs no exchange, the norm one
// sum over the lanes.  P = 8, 16-byte loads, 32-byte ones of FP32; 4 where halves are no multiple of 8 channels.  The pieces of the lanes follow one another in
// memory (FP32, neighbours, 5001 tokens of 16 / 16 heads of 128: with two pieces of a lane in a row and 16-byte loads 39.7 us, so 31.9: 5.8 TB/s; all times in a graph).  The angles are the same for
// all heads: each is worked out by one thread of the block, in 64 bits up to the fraction of a turn (position times frequency in 32 bits would be off by 0.01 rad at position
// 131 072), while the first vectors are on their way, and handed over in shared memory; its sine and cosine are those of the full-precision function (the fast ones: the same times,
// but 120 000 tokens of 1 / 1 heads, where an angle serves two vectors only, 76.3 -> 77.2).
// The threads of a block are dealt to tokens, and a thread stays with its token: the weights of a projection stay in its registers, packed FP32
// pairs do the arithmetic.  Decode steps: a block of 256 threads per token (one of 128: 2.0 -> 2.2 us); prompts: 128 threads, 4 tokens of a block (2 at head_dim 128), so that all
// lanes have several vectors, the next one under way while one is worked on.  What is left above the copy rate are instructions, 14 for a channel.  us, 32 / 8 heads
// of 128: 8192 tokens in bfloat16 with norms 51.1 -> 38.1 (5.3 TB/s), in FP32 51.3 (5.9 TB/s), 1024 tokens 6.5; one token of 32 / 4 heads of 64 2.1.  Of 8192 tokens: 256 threads with twice the
// tokens 39.4, 64 threads 37.8 (but 1024 tokens 8.7), two vectors under way 41.3, other register bounds 42 to 46, sines and cosines in registers (fewer threads) 42.6, with their negatives
// in a third table 41.5.
#include "sa_rotate.cuh"

namespace sa {

// TOKENS: of a block.  NEIGHBOURS: how channels pair.
template <int D, typename T, int P, int TOKENS, bool NEIGHBOURS>
__global__ void __launch_bounds__(rotate_threads(TOKENS), (sizeof(T) == 4 ? 3 : 4) * 256 / rotate_threads(TOKENS)) rotate_kernel(const __grid_constant__ RotateArgs a) {
    __shared__ __align__(16) float turn[TOKENS][2][kRotateMost];
    const int64_t token0 = (int64_t)blockIdx.x * TOKENS;
    pdl_wait();                                                                    // the projections may come from the kernel before
    rotate_tokens<D, T, P, TOKENS, NEIGHBOURS>(a, turn, token0, 0, TOKENS == 1 ? 1 : (int)min((int64_t)TOKENS, a.n - token0),
                                               [&](int kind, int head, int, int64_t token) { return a.out[kind] + (token * a.heads[kind] + head) * D; });
    // a decode kernel behind this one reads its queries before it waits for it
    __threadfence();
}

template <int D, typename T, int P, bool NEIGHBOURS>
static void launch_rotate(const RotateArgs& a, cudaStream_t s) {
    constexpr int kTokens = D == 64 ? 4 : 2;
    // one wave of blocks with a token each, while they fit: 32 / 8 heads of 128, 256 tokens 3.8 us (4.8 with blocks of several), 513 4.7 (5.5), 700 7.4 (5.9)
    if (a.n <= (int64_t)sm_count() * (sizeof(T) == 4 ? 3 : 4)) (void)launch_pdl(rotate_kernel<D, T, P, 1, NEIGHBOURS>, dim3((unsigned)a.n), dim3(rotate_threads(1)), 0, s, a);
    else (void)launch_pdl(rotate_kernel<D, T, P, kTokens, NEIGHBOURS>, dim3((unsigned)((a.n + kTokens - 1) / kTokens)), dim3(rotate_threads(kTokens)), 0, s, a);
}
template <int D, typename T>
static void launch_rotate(const RotateArgs& a, cudaStream_t s) {
    if (a.neighbours) launch_rotate<D, T, 8, true>(a, s);
    else if (a.R % 16 == 0) launch_rotate<D, T, 8, false>(a, s);
    else launch_rotate<D, T, 4, false>(a, s);
}

sa_status rotate_args(const Plan& p, const sa_rotary* rot, const void* const (&in)[3], const int64_t (&stride)[3], uint16_t* const (&out)[3], bool to_cache,
                      const int32_t* positions, int64_t n, RotateArgs* args) {
    if (!rot || n < 0) return SA_ERR_INVALID_ARG;
    if (rot->dtype != SA_F16 && rot->dtype != SA_BF16 && rot->dtype != SA_F32) return SA_ERR_UNSUPPORTED;
    if (rot->rotary_dim < 0 || rot->rotary_dim > p.d || rot->rotary_dim % 8 != 0) return SA_ERR_UNSUPPORTED;
    if (rot->pairs != SA_PAIR_HALVES && rot->pairs != SA_PAIR_NEIGHBOURS) return SA_ERR_INVALID_ARG;
    if (rot->n_axes < 1 || rot->n_axes > 4 || (rot->norm != 0 && rot->norm != 1) || !(rot->eps >= 0.0f)) return SA_ERR_INVALID_ARG;
    if (rot->rotary_dim && (!rot->inv_freq || (rot->n_axes > 1 && !rot->pair_axis))) return SA_ERR_INVALID_ARG;
    RotateArgs a{};
    const int size = rot->dtype == SA_F32 ? 4 : 2;
    int total = 0;
    for (int i = 0; i < 3; ++i) {
        const bool row = i == 0 || !to_cache;
        if (row ? !in[i] != !out[i] : !in[i]) return SA_ERR_INVALID_ARG;
        if (!in[i]) continue;
        a.heads[i] = i == 0 ? p.Hq : p.Hkv;
        if (n > 1 && stride[i] < (int64_t)a.heads[i] * p.d) return SA_ERR_INVALID_ARG;       // rows that overlap
        if (!aligned(in[i], 16) || (row && !aligned(out[i], 16)) || (n > 1 && stride[i] * size % 16 != 0)) return SA_ERR_ALIGNMENT;
        a.in[i] = in[i];
        a.out[i] = row ? out[i] : nullptr;
        a.stride[i] = stride[i];
        a.wide |= (aligned(in[i], 32) && (n == 1 || stride[i] * size % 32 == 0) ? 1 : 0) << i;
        total += a.heads[i];
    }
    if (total == 0) return SA_ERR_INVALID_ARG;
    if (rot->rotary_dim && !positions) return SA_ERR_INVALID_ARG;
    if (!aligned(rot->q_weight, 16) || !aligned(rot->k_weight, 16) || !aligned(rot->inv_freq, 4) || !aligned(positions, 4)) return SA_ERR_ALIGNMENT;
    if (n > 0x7fffffffLL) return SA_ERR_CAPACITY;
    a.weight[0] = rot->q_weight;
    a.weight[1] = rot->k_weight;
    a.positions = positions;
    a.inv_freq = rot->inv_freq;
    a.pair_axis = rot->pair_axis;
    a.n = n;
    a.R = rot->rotary_dim;
    a.axes = rot->n_axes;
    a.norm = rot->norm;
    a.neighbours = rot->pairs == SA_PAIR_NEIGHBOURS;
    a.eps = rot->eps;
    a.scale = rot->scale;
    *args = a;
    return SA_OK;
}

}  // namespace sa

using namespace sa;

extern "C" sa_status sa_rotate_qkv(const sa_config* cfg, const sa_rotary* rot, const void* Q, int64_t q_stride, const void* K, int64_t k_stride,
                                   const void* V, int64_t v_stride, const int32_t* positions, int64_t n, uint16_t* Q_out, uint16_t* K_out,
                                   uint16_t* V_out, sa_stream stream) {
    Plan p;
    sa_status st = make_plan(cfg, &p);
    if (st != SA_OK) return st;
    RotateArgs a;
    st = rotate_args(p, rot, {Q, K, V}, {q_stride, k_stride, v_stride}, {Q_out, K_out, V_out}, false, positions, n, &a);
    if (st != SA_OK || n == 0) return st;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    if (p.d == 64) {
        if (rot->dtype == SA_F16) launch_rotate<64, __half>(a, s);
        else if (rot->dtype == SA_BF16) launch_rotate<64, __nv_bfloat16>(a, s);
        else launch_rotate<64, float>(a, s);
    } else {
        if (rot->dtype == SA_F16) launch_rotate<128, __half>(a, s);
        else if (rot->dtype == SA_BF16) launch_rotate<128, __nv_bfloat16>(a, s);
        else launch_rotate<128, float>(a, s);
    }
    return cudaGetLastError() == cudaSuccess ? SA_OK : SA_ERR_CUDA;
}
