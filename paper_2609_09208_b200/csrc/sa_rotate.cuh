// The step from a layer's projections to binary16 rows (norms of queries and keys, rotation by the position, conversion), for a block of threads: of
// sa_rotate_qkv, whose comment says how the threads are dealt, and of sa_append_qkv.
#pragma once
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

// The block's tokens token0 + first_slot .. token0 + end_slot - 1; row_of(kind, head, slot, token): where the row goes.  TOKENS: of a block.  NEIGHBOURS: how
// channels pair.  turn: scale * cos, scale * sin of every pair.
template <int D, typename T, int P, int TOKENS, bool NEIGHBOURS, typename RowOf>
SA_D void rotate_tokens(const RotateArgs& a, float (&turn)[TOKENS][2][kRotateMost], int64_t token0, int first_slot, int end_slot, RowOf row_of) {
    constexpr int L = D / (2 * P), THREADS = rotate_threads(TOKENS) / TOKENS, GROUPS = THREADS / L, H = P / 2;   // lanes of a vector; threads, vectors of a token
    const int slot = TOKENS == 1 ? 0 : threadIdx.x / THREADS, l = threadIdx.x % L, half = a.R / 2;
    const int64_t token = token0 + slot;
    const int pa = NEIGHBOURS || P * l < half ? P * l : a.R + P * l - half;                                          // first channels of the pieces
    const int pb = NEIGHBOURS ? D / 2 + P * l : P * l < half ? P * l + half : (a.R + D) / 2 + P * l - half;
    const uint32_t mine = ((1u << L) - 1u) << (threadIdx.x & 31 & ~(L - 1));       // the lanes of this vector
    const int per = slot >= first_slot && slot < end_slot ? a.heads[0] + a.heads[1] + a.heads[2] : 0;
    Piece<T, P> one, two;
    auto kind_of = [&](int v) { return v < a.heads[0] ? 0 : v < a.heads[0] + a.heads[1] ? 1 : 2; };
    auto head_of = [&](int v, int kind) { return v - (kind == 0 ? 0 : kind == 1 ? a.heads[0] : a.heads[0] + a.heads[1]); };
    auto load = [&](int v) {                                                       // vector v of the token
        const int kind = kind_of(v);
        const T* in = static_cast<const T*>(a.in[kind]) + token * a.stride[kind] + head_of(v, kind) * D;
        const bool wide = a.wide >> kind & 1;
        one.load(in + pa, wide);
        two.load(in + pb, wide);
    };
    int v = threadIdx.x % THREADS / L;
    if (v < per) load(v);
    const int tokens = TOKENS == 1 ? 1 : end_slot - first_slot;
    for (int i = threadIdx.x; i < half * tokens; i += rotate_threads(TOKENS)) {
        const int j = TOKENS == 1 ? i : i % half, k = TOKENS == 1 ? 0 : first_slot + i / half;
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
        one.get(x);
        two.get(y);
        uint16_t* out = row_of(kind, head_of(v, kind), slot, token);
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
}

// Checks of what a caller gives, and the kernel's arguments (sa_rotate.cu).  to_cache: keys and values have no rows to go to.
sa_status rotate_args(const Plan& p, const sa_rotary* rot, const void* const (&in)[3], const int64_t (&stride)[3], uint16_t* const (&out)[3], bool to_cache,
                      const int32_t* positions, int64_t n, RotateArgs* args);

}  // namespace sa
