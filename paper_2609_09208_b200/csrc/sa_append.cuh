// sa_append_qkv: from a layer's projections to queries and, behind what the cache holds, to its codes: the kernel.
//
// A block takes the tokens of 1, 2 or 4 neighbouring places of a page, all heads: norms, rotation and conversion as sa_rotate_qkv has them (rotate_tokens),
// queries to their rows; keys and values wait in shared memory as the binary16 rows that they would have been, and are coded from there, D / 16 lanes a
// vector, a lane a block of 16 channels: no trip of theirs through memory, and no second launch.  The places a block takes start at a multiple of their
// number, wherever the sequence ends, so that a byte which two tokens share (4-bit values) belongs to one lane.
//
// What bounds it (in a CUDA graph): long chunks memory and the way there (projections in, queries and codes out; a block loads, waits and codes without overlap): 4 chunks of up to 5001
// tokens, 32 / 8 heads of 128, FP32 to rotated INT8 codes 77 us for 349 MB, 69 % of the copy rate (sa_rotate_qkv and sa_fill_kv would move the keys and values twice more).  Few tokens: a launch of 2.3 us and one latency after another, length, page,
// projections, rotation, codes: one token 4.3 us, 32 single tokens 8.2, a chunk of 2048 (with the launch that moves the lengths) 9.2.
#pragma once
#include "sa_cache_write.cuh"
#include "sa_common.cuh"
#include "sa_fp4.cuh"
#include "sa_rotate.cuh"

namespace sa {

constexpr int kAppendBatch = 64;          // sequences per launch
constexpr int kAppendRowsMost = 200 * 1024;      // bytes of keys and values that wait in shared memory
struct AppendSeqs {
    int64_t row0[kAppendBatch];           // first row of the sequence's new tokens
    int tokens[kAppendBatch];
    int blocks[kAppendBatch + 1];         // blocks ahead of it
    int b0, n;                            // sequences b0 .. b0 + n - 1
};
// How keys are stored.  (a.k: mantissa bits of the power-of-two codes.)
enum AppendForm { APPEND_BYTE, APPEND_DENSE, APPEND_INT8, APPEND_FP16, APPEND_FP4 };
struct AppendArgs {
    RotateArgs r;
    CacheArgs c;
    AppendSeqs s;
    int form, bump;                       // bump: the lengths grow here (every sequence has one block)
};

// Whether the pages of tokens start .. start + n - 1 of sequence b are all mapped; by `threads` threads, each of which sees a part.
SA_D bool append_pages(const CacheArgs& c, int b, int start, int n, int thread, int threads) {
    if (start < 0 || n > 0x7fffffff - start) return false;
    bool ok = true;
    for (int lp = start / kPageTokens + thread; lp <= (start + n - 1) / kPageTokens; lp += threads) ok &= page_block(c, b, lp, 0) != nullptr;
    return ok;
}

// 16 channels (pairs of binary16) of a key whose largest magnitude has the bits `top`: a byte a channel.
template <bool INT8>
SA_D void append_bytes(const uint32_t (&x)[8], uint32_t top, int K, uint32_t (&w)[4]) {
    const KeyScale ks = key_scale(top);
    const float amax = half_bits_to_float(top), inv8 = INT8 && top ? __fdiv_rn(127.0f, amax) : 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        w[i] = 0u;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&x[2 * i + k / 2]));
            const float e = k & 1 ? f.y : f.x;
            if constexpr (INT8) {
                const int q = __float2int_rn(__fmul_rn(e, inv8));
                w[i] |= ((uint32_t)max(-127, min(127, q)) & 0xffu) << (8 * k);
            } else {
                uint32_t p = encode_place(K, e, ks);
                p = p < (1u << K) ? 0u : p;
                w[i] |= (((p << (7 - K)) & (0x7fu & (0x7fu << (7 - K)))) | (p >> K)) << (8 * k);
            }
        }
        if constexpr (!INT8) w[i] |= __byte_perm(x[2 * i], x[2 * i + 1], 0x7531) & 0x80808080u & (w[i] + 0x7f7f7f7fu);
    }
}
// ... a nibble a channel, and up to two bits of the mantissa, plane by plane.
SA_D void append_nibbles(const uint32_t (&x)[8], uint32_t top, int K, uint32_t (&w)[2], uint32_t (&plane)[2]) {
    const KeyScale ks = key_scale(top);
    plane[0] = plane[1] = 0u;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        w[i] = 0u;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t h = x[4 * i + e / 2] >> (16 * (e & 1)) & 0xffffu;
            uint32_t p = encode_place(K, half_bits_to_float(h), ks);
            p = p < (1u << K) ? 0u : p;
            const uint32_t g = p >> K;
            w[i] |= (g | (g ? h >> 12 & 8u : 0u)) << (4 * e);
            plane[0] |= (p & (K > 0 ? 1u : 0u)) << (8 * i + e);
            plane[1] |= (p >> 1 & (K > 1 ? 1u : 0u)) << (8 * i + e);
        }
    }
}
// ... of a value: INT8 times 2^-g.
SA_D void append_values(const uint32_t (&x)[8], int g, uint32_t (&w)[4]) {
    const float f = pow2i(g);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        // scaling by 2^g is exact, so adding 1.5 * 2^23 rounds to the nearest integer (ties to even), the low byte of the bits
        const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&x[2 * i])), b = __half22float2(*reinterpret_cast<const __half2*>(&x[2 * i + 1]));
        const uint32_t lo = __byte_perm(__float_as_uint(__fmaf_rn(a.x, f, 12582912.0f)), __float_as_uint(__fmaf_rn(a.y, f, 12582912.0f)), 0x0040);
        const uint32_t hi = __byte_perm(__float_as_uint(__fmaf_rn(b.x, f, 12582912.0f)), __float_as_uint(__fmaf_rn(b.y, f, 12582912.0f)), 0x0040);
        w[i] = __byte_perm(lo, hi, 0x5410);
    }
}

// Codes the rows of tokens first .. end - 1 of the block's places (place 0 is token t0 of its half page at `halves` + head * page_bytes).
template <int D, int TOKENS, int THREADS>
SA_D void append_codes(const CacheArgs& c, int form, uint8_t* halves, int t0, int first, int end, const uint16_t* rows) {
    constexpr int LPV = D / 16, VECTORS = THREADS / LPV;
    const Fp4Half<D> f(threadIdx.x & 31, 0);
    const int mine = threadIdx.x / LPV, blk = f.blk;
    auto row_of = [&](int place, int values, int head) { return rows + ((size_t)(place * 2 + values) * c.Hkv + head) * D + 16 * blk; };
    auto load = [&](const uint16_t* p, uint32_t (&x)[8]) {
        const uint4 a = reinterpret_cast<const uint4*>(p)[0], b = reinterpret_cast<const uint4*>(p)[1];
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    };
    auto largest = [&](const uint32_t (&x)[8]) {                      // of the whole vector
        uint32_t top = x[0] & 0x7fff7fffu;
#pragma unroll
        for (int e = 1; e < 8; ++e) top = __vmaxu2(top, x[e] & 0x7fff7fffu);
        top = max(top & 0xffffu, top >> 16);
#pragma unroll
        for (int o = 1; o < LPV; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
        return top;
    };
    const int keys = (end - first) * c.Hkv;
#pragma unroll 1
    for (int i0 = 0; i0 < keys; i0 += VECTORS) {                      // (whole warps: the lanes of a vector exchange numbers)
        const int i = min(i0 + mine, keys - 1), place = first + i / c.Hkv, head = i % c.Hkv, t = t0 + place;
        const bool there = i0 + mine < keys;
        uint8_t* half = halves + (size_t)head * c.page_bytes;
        uint32_t x[8];
        load(row_of(place, 0, head), x);
        if (c.hadamard) f.rotate(x);
        if (form == APPEND_FP16) {
            uint4* to = reinterpret_cast<uint4*>(half + c.kcode_off) + 2 * blk * kTileTokens + t;
            if (there) {
                to[0] = make_uint4(x[0], x[1], x[2], x[3]);
                to[kTileTokens] = make_uint4(x[4], x[5], x[6], x[7]);
            }
        } else if (form == APPEND_FP4) {
            uint32_t w[2];
            const uint32_t scale = fp4_block(x, w);
            if (there) {
                *reinterpret_cast<uint32_t*>(half + fp4_key_byte(t, 16 * blk)) = w[0];
                *reinterpret_cast<uint32_t*>(half + fp4_key_byte(t, 16 * blk + 8)) = w[1];
                half[fp4_key_scale(D, t, 16 * blk)] = (uint8_t)scale;
            }
        } else {
            const uint32_t top = largest(x);
            if (form == APPEND_DENSE) {
                uint32_t w[2], plane[2];
                append_nibbles(x, top, c.k, w, plane);
                if (there) {
                    *reinterpret_cast<uint2*>(half + c.kcode_off + (size_t)(blk / 2 * kTileTokens + t) * 16 + blk % 2 * 8) = make_uint2(w[0], w[1]);
                    for (int bit = 0; bit < c.k; ++bit)
                        *reinterpret_cast<uint16_t*>(half + c.plane_off + (size_t)(bit * kTileTokens + t) * (D / 8) + 2 * blk) = (uint16_t)plane[bit];
                }
            } else {
                uint32_t w[4];
                if (form == APPEND_INT8) append_bytes<true>(x, top, 0, w);
                else append_bytes<false>(x, top, c.k, w);
                if (there) *reinterpret_cast<uint4*>(half + c.kcode_off + (size_t)(blk * kTileTokens + t) * 16) = make_uint4(w[0], w[1], w[2], w[3]);
            }
            if (there && blk == 0) *reinterpret_cast<uint16_t*>(half + c.meta_off + (size_t)t * 4) = (uint16_t)top;
        }
    }
    if (form == APPEND_FP4) {
        // values by pairs of tokens: a byte has a nibble of either; where one of them is not new, its nibble stays
        const int pair0 = (t0 + first) / 2, pairs = ((t0 + end - 1) / 2 - pair0 + 1) * c.Hkv;
#pragma unroll 1
        for (int i = mine; i < pairs; i += VECTORS) {
            const int head = i % c.Hkv, t = (pair0 + i / c.Hkv) * 2;
            uint8_t* v = halves + (size_t)head * c.page_bytes + c.v_off;
            uint32_t w[2][2] = {}, mask = 0;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int place = t + k - t0;
                if (place < first || place >= end) continue;
                uint32_t x[8];
                load(row_of(place, 1, head), x);
                v[fp4_value_scale(D, t + k, 16 * blk)] = (uint8_t)fp4_block(x, w[k]);
                mask |= k ? 0xf0f0u : 0x0f0fu;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {                             // channels e and e + 8 of the block: two bytes
                auto nibble = [&](uint32_t word) { return word >> (4 * e) & 15u; };
                uint32_t x = nibble(w[0][0]) | nibble(w[1][0]) << 4 | nibble(w[0][1]) << 8 | nibble(w[1][1]) << 12;
                uint16_t* at = reinterpret_cast<uint16_t*>(v + fp4_value_byte(t, 16 * blk + e));
                if (mask != 0xffffu) x |= *at & ~mask;
                *at = (uint16_t)x;
            }
        }
        return;
    }
#pragma unroll 1
    for (int i0 = 0; i0 < keys; i0 += VECTORS) {
        const int i = min(i0 + mine, keys - 1), place = first + i / c.Hkv, head = i % c.Hkv, t = t0 + place;
        const bool there = i0 + mine < keys;
        uint8_t* half = halves + (size_t)head * c.page_bytes;
        uint32_t x[8];
        load(row_of(place, 1, head), x);
        if (form == APPEND_FP16) {
            uint4* to = reinterpret_cast<uint4*>(half + c.v_off) + 2 * blk * kTileTokens + t;
            if (there) {
                to[0] = make_uint4(x[0], x[1], x[2], x[3]);
                to[kTileTokens] = make_uint4(x[4], x[5], x[6], x[7]);
            }
        } else {
            const int g = value_exponent(largest(x));
            uint32_t w[4];
            append_values(x, g, w);
            if (there) {
                *reinterpret_cast<uint4*>(half + c.v_off + (size_t)(blk * kTileTokens + t) * 16) = make_uint4(w[0], w[1], w[2], w[3]);
                if (blk == 0) *reinterpret_cast<uint16_t*>(half + c.meta_off + (size_t)t * 4 + 2) = (uint16_t)(g & 0xff);
            }
        }
    }
}

template <int D, typename T, int P, int TOKENS, bool NEIGHBOURS>
__global__ void __launch_bounds__(rotate_threads(TOKENS), (sizeof(T) == 4 ? 3 : 4) * 256 / rotate_threads(TOKENS)) append_qkv_kernel(const __grid_constant__ AppendArgs a) {
    __shared__ __align__(16) float turn[TOKENS][2][kRotateMost];
    extern __shared__ uint4 dynamic[];
    uint16_t* rows = reinterpret_cast<uint16_t*>(dynamic);                             // [place][keys, values][head][D]
    const int lane = threadIdx.x & 31, block = blockIdx.x;
    int i = 0;                                                                         // the sequence: the last one that starts at or before the block
    for (int j0 = 0; j0 < a.s.n; j0 += 32) {
        const int j = j0 + lane;
        i += __popc(__ballot_sync(0xffffffffu, j < a.s.n && a.s.blocks[j + 1] <= block));
    }
    const int b = a.s.b0 + i, n = a.s.tokens[i];
    pdl_wait();                                                                        // earlier kernels may read this cache or write the inputs
    const int start = a.c.seq_lens[b];
    // A length that cannot be one: queries go to their rows all the same.
    const int64_t from = max(start, 0), place0 = (from / TOKENS + block - a.s.blocks[i]) * TOKENS;
    const int first = (int)max(from - place0, (int64_t)0), end = (int)min(from + n - place0, (int64_t)TOKENS);
    const bool ok = __syncthreads_and(append_pages(a.c, b, start, n, threadIdx.x, rotate_threads(TOKENS)));       // (every thread has read the length before it changes)
    if (first >= end) return;
    rotate_tokens<D, T, P, TOKENS, NEIGHBOURS>(a.r, turn, a.s.row0[i] + place0 - from, first, end, [&](int kind, int head, int slot, int64_t token) {
        return kind == 0 ? a.r.out[0] + (token * a.r.heads[0] + head) * D : rows + ((size_t)(slot * 2 + kind - 1) * a.c.Hkv + head) * D;
    });
    __syncthreads();
    if (ok) {
        const int t = (int)(place0 % kPageTokens);                                     // (the block's places lie in one half page)
        uint8_t* page = page_block(a.c, b, (int)(place0 / kPageTokens), 0);
        append_codes<D, TOKENS, rotate_threads(TOKENS)>(a.c, a.form, page + (size_t)(t >> 5) * (a.c.page_bytes >> 1), t & 31, first, end, rows);
        if (a.bump && threadIdx.x == 0) a.c.seq_lens[b] = start + n;
    }
    // a decode kernel behind this one reads its queries before it waits for it
    __threadfence();
}

template <int D, typename T, int P, bool NEIGHBOURS>
cudaError_t launch_append(const AppendArgs& a, int tokens, cudaStream_t s) {
    constexpr int kTokens = D == 64 ? 4 : 2;
    const int rows = (int)sizeof(uint16_t) * 2 * a.c.Hkv * D;
    const unsigned grid = (unsigned)a.s.blocks[a.s.n];
    // The most that any call needs, not this one's rows: it is asked for once, and the kernel's sines and cosines count against the 48 KB that need no asking.
    if (tokens == 1) {
        static OncePerDevice once;
        if (!allow_shared(append_qkv_kernel<D, T, P, 1, NEIGHBOURS>, kAppendRowsMost, once)) return cudaGetLastError();
        return launch_pdl(append_qkv_kernel<D, T, P, 1, NEIGHBOURS>, dim3(grid), dim3(rotate_threads(1)), (size_t)rows, s, a);
    }
    static OncePerDevice once;
    if (!allow_shared(append_qkv_kernel<D, T, P, kTokens, NEIGHBOURS>, kAppendRowsMost, once)) return cudaGetLastError();
    return launch_pdl(append_qkv_kernel<D, T, P, kTokens, NEIGHBOURS>, dim3(grid), dim3(rotate_threads(kTokens)), (size_t)kTokens * rows, s, a);
}
template <int D, typename T>
cudaError_t launch_append(const AppendArgs& a, int tokens, cudaStream_t s) {
    if (a.r.neighbours) return launch_append<D, T, 8, true>(a, tokens, s);
    if (a.r.R % 16 == 0) return launch_append<D, T, 8, false>(a, tokens, s);
    return launch_append<D, T, 4, false>(a, tokens, s);
}
template <typename T>
cudaError_t launch_append_typed(const AppendArgs& a, int d, int tokens, cudaStream_t s) {
    return d == 64 ? launch_append<64, T>(a, tokens, s) : launch_append<128, T>(a, tokens, s);
}
// (sa_append_f32.cu, sa_append_bf16.cu, sa_append.cu)
cudaError_t launch_append_f32(const AppendArgs& a, int d, int tokens, cudaStream_t s);
cudaError_t launch_append_bf16(const AppendArgs& a, int d, int tokens, cudaStream_t s);

}  // namespace sa
