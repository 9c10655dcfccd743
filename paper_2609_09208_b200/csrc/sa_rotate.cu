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
#include "sa_cache_write.cuh"
#include "sa_common.cuh"
#include <cuda_bf16.h>
#include <type_traits>

namespace sa {

struct RotateArgs {
    const void* in[3];                    // queries, keys, values; rows of a token
    int64_t stride[3];                    // elements from one token's row to the next
    uint16_t* out[3];
    const void* weight[2];
    const int32_t* positions;             // [axes][n]
    const float* inv_freq;                // [R / 2]
    const uint8_t* pair_axis;             // [R / 2] or null
    int64_t n;
    int heads[3], R, axes, norm, neighbours;
    int wide;                             // bit i: rows of in[i] start on 32-byte boundaries
    float eps, scale;
};
SA_HD constexpr int rotate_threads(int tokens) { return tokens == 1 ? 256 : 128; }
constexpr int kRotateMost = 64;           // pairs

// P channels as they lie in memory, and as pairs of FP32.
template <typename T, int P>
struct Piece {
    static constexpr int kWords = P * (int)sizeof(T) / 4;
    uint32_t w[kWords];
    SA_D void load(const T* p, bool wide) {                   // wide: p is a multiple of 32 bytes
        if constexpr (kWords == 8) load_32_bytes(p, wide, w);
        else if constexpr (kWords == 2) {
            const uint2 v = *reinterpret_cast<const uint2*>(p);
            w[0] = v.x, w[1] = v.y;
        } else
#pragma unroll
            for (int i = 0; i < kWords; i += 4) {
                const uint4 v = reinterpret_cast<const uint4*>(p)[i / 4];
                w[i] = v.x, w[i + 1] = v.y, w[i + 2] = v.z, w[i + 3] = v.w;
            }
    }
    SA_D void get(f32x2 (&x)[P / 2]) const {
#pragma unroll
        for (int i = 0; i < P / 2; ++i) {
            if constexpr (sizeof(T) == 4) x[i] = pack_f32x2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
            else if constexpr (std::is_same_v<T, __half>) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
                x[i] = pack_f32x2(f.x, f.y);
            } else x[i] = pack_f32x2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));      // bfloat16: the upper half of an FP32 number
        }
    }
};
template <int P>
SA_D void store_halves(uint16_t* p, const f32x2 (&x)[P / 2]) {
    uint32_t h[P / 2];
#pragma unroll
    for (int i = 0; i < P / 2; ++i) {
        float lo, hi;
        unpack_f32x2(x[i], &lo, &hi);
        const __half2 v = __floats2half2_rn(lo, hi);
        h[i] = *reinterpret_cast<const uint32_t*>(&v);
    }
    if constexpr (P == 8) *reinterpret_cast<uint4*>(p) = make_uint4(h[0], h[1], h[2], h[3]);
    else *reinterpret_cast<uint2*>(p) = make_uint2(h[0], h[1]);
}

// TOKENS: of a block.  NEIGHBOURS: how channels pair.
template <int D, typename T, int P, int TOKENS, bool NEIGHBOURS>
__global__ void __launch_bounds__(rotate_threads(TOKENS), (sizeof(T) == 4 ? 3 : 4) * 256 / rotate_threads(TOKENS)) rotate_kernel(const __grid_constant__ RotateArgs a) {
    constexpr int L = D / (2 * P), THREADS = rotate_threads(TOKENS) / TOKENS, GROUPS = THREADS / L, H = P / 2;   // lanes of a vector; threads, vectors of a token
    __shared__ __align__(16) float turn[TOKENS][2][kRotateMost];                               // scale * cos, scale * sin of every pair
    const int64_t token0 = (int64_t)blockIdx.x * TOKENS;
    const int slot = TOKENS == 1 ? 0 : threadIdx.x / THREADS, l = threadIdx.x % L, half = a.R / 2;
    const int64_t token = token0 + slot;
    const int pa = NEIGHBOURS || P * l < half ? P * l : a.R + P * l - half;                                          // first channels of the pieces
    const int pb = NEIGHBOURS ? D / 2 + P * l : P * l < half ? P * l + half : (a.R + D) / 2 + P * l - half;
    const uint32_t mine = ((1u << L) - 1u) << (threadIdx.x & 31 & ~(L - 1));       // the lanes of this vector
    const int per = token < a.n ? a.heads[0] + a.heads[1] + a.heads[2] : 0;
    Piece<T, P> first, second;
    auto kind_of = [&](int v) { return v < a.heads[0] ? 0 : v < a.heads[0] + a.heads[1] ? 1 : 2; };
    auto head_of = [&](int v, int kind) { return v - (kind == 0 ? 0 : kind == 1 ? a.heads[0] : a.heads[0] + a.heads[1]); };
    auto load = [&](int v) {                                                       // vector v of the token
        const int kind = kind_of(v);
        const T* in = static_cast<const T*>(a.in[kind]) + token * a.stride[kind] + head_of(v, kind) * D;
        const bool wide = a.wide >> kind & 1;
        first.load(in + pa, wide);
        second.load(in + pb, wide);
    };
    int v = threadIdx.x % THREADS / L;
    pdl_wait();                                                                    // the projections may come from the kernel before
    if (v < per) load(v);
    const int tokens = TOKENS == 1 ? 1 : (int)min((int64_t)TOKENS, a.n - token0);
    for (int i = threadIdx.x; i < half * tokens; i += rotate_threads(TOKENS)) {
        const int j = TOKENS == 1 ? i : i % half, k = TOKENS == 1 ? 0 : i / half;
        const int axis = a.pair_axis ? min((int)a.pair_axis[j], a.axes - 1) : 0;
        const double turns = (double)a.positions[axis * a.n + token0 + k] * (double)a.inv_freq[j] * 0.15915494309189535;
        // the fraction's sine and cosine to their last bits: one channel of a pair may be far larger than the other
        float sn, cs;
        sincospif(2.0f * (float)(turns - rint(turns)), &sn, &cs);
        turn[k][0][j] = cs * a.scale;
        turn[k][1][j] = sn * a.scale;
    }
    __syncthreads();
    const bool turns_a = pa < (NEIGHBOURS ? a.R : half), turns_b = NEIGHBOURS ? pb < a.R : turns_a;
    // from shared memory for every vector: in registers they would cost a third of the threads, and with them of the bytes under way
    const float *ca = turn[slot][0] + (NEIGHBOURS ? pa / 2 : pa), *sa = turn[slot][1] + (NEIGHBOURS ? pa / 2 : pa);
    const float *cb = turn[slot][0] + pb / 2, *sb = turn[slot][1] + pb / 2;
    Piece<T, P> wa, wb;
    int weights_of = -1;
    while (v < per) {
        const int kind = kind_of(v);
        f32x2 x[H], y[H];
        first.get(x);
        second.get(y);
        uint16_t* out = a.out[kind] + (token * a.heads[kind] + head_of(v, kind)) * D;
        v += GROUPS;
        if (v < per) load(v);                                                      // (the next vector is under way while this one is worked on)
        if (kind < 2) {
            if (a.norm) {
                f32x2 sum2 = mul2(x[0], x[0]);
#pragma unroll
                for (int i = 1; i < H; ++i) sum2 = ffma2(x[i], x[i], sum2);
#pragma unroll
                for (int i = 0; i < H; ++i) sum2 = ffma2(y[i], y[i], sum2);
                float lo, hi;
                unpack_f32x2(sum2, &lo, &hi);
                float sum = lo + hi;
#pragma unroll
                for (int o = 1; o < L; o <<= 1) sum += __shfl_xor_sync(mine, sum, o);
                const float r = rsqrtf(sum * (1.0f / D) + a.eps);
                const f32x2 rr = pack_f32x2(r, r);
                if (weights_of != kind && a.weight[kind]) {
                    weights_of = kind;
                    wa.load(static_cast<const T*>(a.weight[kind]) + pa, false);
                    wb.load(static_cast<const T*>(a.weight[kind]) + pb, false);
                }
#pragma unroll
                for (int i = 0; i < H; ++i) {
                    x[i] = mul2(x[i], rr);
                    y[i] = mul2(y[i], rr);
                }
                if (a.weight[kind]) {
                    f32x2 w[H];
                    wa.get(w);
#pragma unroll
                    for (int i = 0; i < H; ++i) x[i] = mul2(x[i], w[i]);
                    wb.get(w);
#pragma unroll
                    for (int i = 0; i < H; ++i) y[i] = mul2(y[i], w[i]);
                }
            }
            if constexpr (NEIGHBOURS) {
                auto rotate = [](f32x2& p, float cs, float sn) {
                    float u, w;
                    unpack_f32x2(p, &u, &w);
                    p = ffma2(pack_f32x2(w, u), pack_f32x2(-sn, sn), mul2(p, pack_f32x2(cs, cs)));
                };
#pragma unroll
                for (int i = 0; i < H; ++i) {
                    if (turns_a) rotate(x[i], ca[i], sa[i]);
                    if (turns_b) rotate(y[i], cb[i], sb[i]);
                }
            } else if (turns_a) {
                const f32x2 minus = pack_f32x2(-1.0f, -1.0f);
#pragma unroll
                for (int i = 0; i < H; ++i) {
                    const f32x2 c = reinterpret_cast<const f32x2*>(ca)[i], t = reinterpret_cast<const f32x2*>(sa)[i];
                    const f32x2 u = ffma2(mul2(y[i], t), minus, mul2(x[i], c));
                    y[i] = ffma2(y[i], c, mul2(x[i], t));
                    x[i] = u;
                }
            }
        }
        store_halves<P>(out + pa, x);
        store_halves<P>(out + pb, y);
    }
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

}  // namespace sa

using namespace sa;

extern "C" sa_status sa_rotate_qkv(const sa_config* cfg, const sa_rotary* rot, const void* Q, int64_t q_stride, const void* K, int64_t k_stride,
                                   const void* V, int64_t v_stride, const int32_t* positions, int64_t n, uint16_t* Q_out, uint16_t* K_out,
                                   uint16_t* V_out, sa_stream stream) {
    Plan p;
    const sa_status st = make_plan(cfg, &p);
    if (st != SA_OK) return st;
    if (!rot || n < 0) return SA_ERR_INVALID_ARG;
    if (rot->dtype != SA_F16 && rot->dtype != SA_BF16 && rot->dtype != SA_F32) return SA_ERR_UNSUPPORTED;
    if (rot->rotary_dim < 0 || rot->rotary_dim > p.d || rot->rotary_dim % 8 != 0) return SA_ERR_UNSUPPORTED;
    if (rot->pairs != SA_PAIR_HALVES && rot->pairs != SA_PAIR_NEIGHBOURS) return SA_ERR_INVALID_ARG;
    if (rot->n_axes < 1 || rot->n_axes > 4 || (rot->norm != 0 && rot->norm != 1) || !(rot->eps >= 0.0f)) return SA_ERR_INVALID_ARG;
    if (rot->rotary_dim && (!rot->inv_freq || (rot->n_axes > 1 && !rot->pair_axis))) return SA_ERR_INVALID_ARG;
    RotateArgs a{};
    const void* in[3] = {Q, K, V};
    const int64_t stride[3] = {q_stride, k_stride, v_stride};
    uint16_t* out[3] = {Q_out, K_out, V_out};
    const int size = rot->dtype == SA_F32 ? 4 : 2;
    int total = 0;
    for (int i = 0; i < 3; ++i) {
        if (!in[i] != !out[i]) return SA_ERR_INVALID_ARG;
        if (!in[i]) continue;
        a.heads[i] = i == 0 ? p.Hq : p.Hkv;
        if (n > 1 && stride[i] < (int64_t)a.heads[i] * p.d) return SA_ERR_INVALID_ARG;       // rows that overlap
        if (!aligned(in[i], 16) || !aligned(out[i], 16) || (n > 1 && stride[i] * size % 16 != 0)) return SA_ERR_ALIGNMENT;
        a.in[i] = in[i];
        a.out[i] = out[i];
        a.stride[i] = stride[i];
        a.wide |= (aligned(in[i], 32) && (n == 1 || stride[i] * size % 32 == 0) ? 1 : 0) << i;
        total += a.heads[i];
    }
    if (total == 0) return SA_ERR_INVALID_ARG;
    if (rot->rotary_dim && !positions) return SA_ERR_INVALID_ARG;
    if (!aligned(rot->q_weight, 16) || !aligned(rot->k_weight, 16) || !aligned(rot->inv_freq, 4) || !aligned(positions, 4)) return SA_ERR_ALIGNMENT;
    if (n == 0) return SA_OK;
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
