// sa_rotate_qkv: from a layer's projections to the rows that the cache and the decode calls take.
//
// One pass over the data: y = x / sqrt(mean(x^2) + eps) * w for every query and key head, then the rotation of its first R channels by
// the token's positions, FP32 throughout, one rounding to binary16; values are converted.  Bound by memory (each input read, each
// output written once); single tokens by latency.
//
// A block takes one token.  d / 8 lanes share a head vector; a lane holds two pieces of four channels whose pairs lie in the lane:
// pairing halves, channels u .. u + 3 and their partners; pairing neighbours, eight channels in a row.  The rotation needs no
// exchange, the norm one sum over the lanes.  The angles are the same for all heads: each is worked out by one thread of the
// block, in 64 bits up to the fraction of a turn (position times frequency in 32 bits would be off by 0.01 rad at position 131 072),
// and handed over in shared memory while the first vectors are on their way.
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
    float eps, scale;
};
constexpr int kRotateThreads = 256;
constexpr int kRotateMost = 64;           // pairs

template <typename T>
SA_D void load4(const T* p, float (&x)[4]) {
    if constexpr (sizeof(T) == 4) {
        const float4 v = *reinterpret_cast<const float4*>(p);
        x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
    } else {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        float2 a, b;
        if constexpr (std::is_same_v<T, __half>) {
            a = __half22float2(*reinterpret_cast<const __half2*>(&v.x));
            b = __half22float2(*reinterpret_cast<const __half2*>(&v.y));
        } else {
            a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&v.x));
            b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&v.y));
        }
        x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y;
    }
}
SA_D void store4(uint16_t* p, const float (&x)[4]) {
    const __half2 a = __floats2half2_rn(x[0], x[1]), b = __floats2half2_rn(x[2], x[3]);
    *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

template <int D, typename T>
__global__ void __launch_bounds__(kRotateThreads) rotate_kernel(const __grid_constant__ RotateArgs a) {
    constexpr int L = D / 8, GROUPS = kRotateThreads / L;                          // lanes of a vector, vectors at a time
    __shared__ float2 turn[kRotateMost];                                           // scale * (cos, sin) of every pair
    const int64_t token = blockIdx.x;
    const int l = threadIdx.x % L, half = a.R / 2;
    const int pa = a.neighbours ? 8 * l : 4 * l < half ? 4 * l : a.R + 4 * l - half;                                 // first channels of the pieces
    const int pb = a.neighbours ? 8 * l + 4 : 4 * l < half ? 4 * l + half : (a.R + D) / 2 + 4 * l - half;
    pdl_wait();                                                                    // the projections may come from the kernel before
    if ((int)threadIdx.x < half) {
        const int j = threadIdx.x, axis = a.pair_axis ? min((int)a.pair_axis[j], a.axes - 1) : 0;
        const double turns = (double)a.positions[axis * a.n + token] * (double)a.inv_freq[j] * 0.15915494309189535;
        float s, c;
        sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
        turn[j] = make_float2(c * a.scale, s * a.scale);
    }
    __syncthreads();
    const uint32_t mine = ((1u << L) - 1u) << (threadIdx.x & 31 & ~(L - 1));       // the lanes of this vector
    const int total = a.heads[0] + a.heads[1] + a.heads[2];
    for (int v = threadIdx.x / L; v < total; v += GROUPS) {
        const int kind = v < a.heads[0] ? 0 : v < a.heads[0] + a.heads[1] ? 1 : 2;
        const int h = kind == 0 ? v : kind == 1 ? v - a.heads[0] : v - a.heads[0] - a.heads[1];
        const T* in = static_cast<const T*>(a.in[kind]) + token * a.stride[kind] + h * D;
        uint16_t* out = a.out[kind] + (token * a.heads[kind] + h) * D;
        float x[4], y[4];
        load4(in + pa, x);
        load4(in + pb, y);
        if (kind < 2) {
            if (a.norm) {
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i) sum += x[i] * x[i] + y[i] * y[i];
#pragma unroll
                for (int o = 1; o < L; o <<= 1) sum += __shfl_xor_sync(mine, sum, o);
                const float r = rsqrtf(sum * (1.0f / D) + a.eps);
                float wx[4] = {1.0f, 1.0f, 1.0f, 1.0f}, wy[4] = {1.0f, 1.0f, 1.0f, 1.0f};
                if (a.weight[kind]) {
                    load4(static_cast<const T*>(a.weight[kind]) + pa, wx);
                    load4(static_cast<const T*>(a.weight[kind]) + pb, wy);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[i] = x[i] * r * wx[i];
                    y[i] = y[i] * r * wy[i];
                }
            }
            if (a.neighbours) {
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    if (pa + i < a.R) {
                        const float2 t = turn[(pa + i) / 2];
                        const float p = x[i], q = x[i + 1];
                        x[i] = p * t.x - q * t.y;
                        x[i + 1] = p * t.y + q * t.x;
                    }
                    if (pb + i < a.R) {
                        const float2 t = turn[(pb + i) / 2];
                        const float p = y[i], q = y[i + 1];
                        y[i] = p * t.x - q * t.y;
                        y[i + 1] = p * t.y + q * t.x;
                    }
                }
            } else if (pa < half) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 t = turn[pa + i];
                    const float p = x[i], q = y[i];
                    x[i] = p * t.x - q * t.y;
                    y[i] = p * t.y + q * t.x;
                }
            }
        }
        store4(out + pa, x);
        store4(out + pb, y);
    }
    // a decode kernel behind this one reads its queries before it waits for it
    __threadfence();
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
    const dim3 grid((unsigned)n), block(kRotateThreads);
#define CALL(D, T) (void)launch_pdl(rotate_kernel<D, T>, grid, block, 0, s, a)
    if (p.d == 64) {
        if (rot->dtype == SA_F16) CALL(64, __half);
        else if (rot->dtype == SA_BF16) CALL(64, __nv_bfloat16);
        else CALL(64, float);
    } else {
        if (rot->dtype == SA_F16) CALL(128, __half);
        else if (rot->dtype == SA_BF16) CALL(128, __nv_bfloat16);
        else CALL(128, float);
    }
#undef CALL
    return cudaGetLastError() == cudaSuccess ? SA_OK : SA_ERR_CUDA;
}
