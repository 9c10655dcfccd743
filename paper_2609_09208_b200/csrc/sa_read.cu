// sa_read_kv: keys and values of a cache back as binary16 rows.
#include "sa_cache_write.cuh"
#include "sa_common.cuh"
#include "sa_score_mma.cuh"

namespace sa {

// One warp takes the keys or the values of one KV head for the 32 tokens of half a page, lane = token, as the fill does: its loads are
// the 16-byte chunks of the half, 512 contiguous bytes each, and the rows are turned in shared memory, so that whole
// 128-byte lines are stored.  Bound by memory: the records read and 2 d bytes written for a key or value.  All of a vector's chunks are asked for at
// once, with as many registers as 9 blocks on an SM leave (8 at head_dim 128): 8 x 16 384 tokens of PoT-M4, 4 heads of 64, 39.4 -> 33.6 us (6.1 TB/s), of 8 x 8192 of INT8
// 21.8 -> 18.4, against a register bound of the compiler's choice and chunks by two; 8 heads of 128, 8192 tokens 13.9 -> 12.7; 11 blocks 37.5 and 20.8.  (Not of 4 bits at head_dim 128: no faster, and a read of the new tokens behind a step takes 0.6 us longer.)
constexpr int kReadBatch = 64;            // sequences per launch
struct ReadSeqs {
    int64_t row0[kReadBatch];             // row of the sequence's first token in K / V
    int tiles[kReadBatch + 1];            // 32-token tiles ahead of it
    int start[kReadBatch], len[kReadBatch];
    int b0, n;
};

SA_D uint32_t half2_bits(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// Walsh-Hadamard rotation of a vector in one thread, as the encoder's; its own inverse.
template <int D>
SA_D void rotate_back(float (&x)[D]) {
#pragma unroll
    for (int st = 1; st < D; st <<= 1)
#pragma unroll
        for (int i = 0; i < D; ++i)
            if ((i & st) == 0) {
                const float a = x[i], b = x[i + st];
                x[i] = __fadd_rn(a, b);
                x[i + st] = __fsub_rn(a, b);
            }
    const float scale = (D == 64) ? 0.125f : 0.088388346f;
#pragma unroll
    for (int i = 0; i < D; ++i) x[i] = __fmul_rn(x[i], scale);
}

// Eight consecutive channels (8 c .. 8 c + 7) of the key of token t in a half, before rounding.  MODE as in write_token.
template <int D, int MODE>
struct KeyReader {
    const uint8_t* half;
    size_t plane_off;
    int t;
    float s;                              // scale of the vector
    uint4 w;                              // the chunk at hand
    SA_D KeyReader(const uint8_t* half_, const CacheArgs& a, int t_) : half(half_), plane_off(a.plane_off), t(t_), s(1.0f) {
        if constexpr (MODE != 16) s = half_bits_to_float(*reinterpret_cast<const uint16_t*>(half + a.meta_off + t * 4));
    }
    SA_D uint4 chunk(int k) const { return load_16_bytes(half + ((size_t)k * kTileTokens + t) * 16); }
    SA_D void get(int c, float (&x)[8]) {
        if constexpr (MODE == 16) {
            w = chunk(c);
            const uint32_t h[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = half_bits_to_float((h[i / 2] >> (16 * (i & 1))) & 0xffffu);
        } else if constexpr (MODE == 32) {                                        // INT8
            if (c % 2 == 0) w = chunk(c / 2);
            const uint32_t h[2] = {c % 2 ? w.z : w.x, c % 2 ? w.w : w.y};
            const f32x2 s2 = pack_f32x2(s, s), d2 = pack_f32x2(-127.0f, -127.0f), i2 = pack_f32x2(1.0f / 127.0f, 1.0f / 127.0f);
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
                const uint32_t even = int8_to_half2<false>(h[i / 4]), odd = int8_to_half2<true>(h[i / 4]);
                const float2 e = __half22float2(*reinterpret_cast<const __half2*>(&even)), o = __half22float2(*reinterpret_cast<const __half2*>(&odd));
                const f32x2 v[2] = {mul2(pack_f32x2(e.x, o.x), s2), mul2(pack_f32x2(e.y, o.y), s2)};       // code times scale: exact
#pragma unroll
                for (int k = 0; k < 2; ++k) {                                     // over 127, as good as rounded correctly
                    const f32x2 q = mul2(v[k], i2);
                    unpack_f32x2(ffma2(ffma2(q, d2, v[k]), i2, q), &x[i + 2 * k], &x[i + 2 * k + 1]);
                }
            }
        } else if constexpr (MODE < 8) {                                          // a byte a channel: bfloat16 numbers, 2^-120 of the codes'
            if (c % 2 == 0) w = chunk(c / 2);
            const uint32_t h[2] = {c % 2 ? w.z : w.x, c % 2 ? w.w : w.y};
            const f32x2 up = pack_f32x2(0x1p120f, 0x1p120f), s2 = pack_f32x2(s, s);
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const uint32_t p = i & 2 ? byte_codes_to_bf16<2>(h[i / 4], 1u) : byte_codes_to_bf16<0>(h[i / 4], 1u);
                unpack_f32x2(mul2(mul2(pack_f32x2(__uint_as_float(p << 16), __uint_as_float(p & 0xffff0000u)), up), s2), &x[i], &x[i + 1]);
            }
        } else {                                                                  // nibbles, and K planes of mantissa bits
            constexpr int K = MODE - 8;
            if (c % 4 == 0) w = chunk(c / 4);
            const uint32_t h = c % 4 == 0 ? w.x : c % 4 == 1 ? w.y : c % 4 == 2 ? w.z : w.w;
            uint32_t plane[K ? K : 1] = {};
#pragma unroll
            for (int bit = 0; bit < K; ++bit) plane[bit] = half[plane_off + ((size_t)bit * kTileTokens + t) * (D / 8) + c];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t b = (h >> (4 * i)) & 15u;
                uint32_t j = 0;
#pragma unroll
                for (int bit = 0; bit < K; ++bit) j |= ((plane[bit] >> i) & 1u) << (4 - K + bit);
                x[i] = power_of_two(b & 7u, 16u + j, b >> 3) * s;
            }
        }
    }
    // sigma * mantissa / 16 * 2^(g - 7); g = 0: the zero code
    SA_D static float power_of_two(uint32_t g, uint32_t mantissa, uint32_t sign) {
        const float f = g ? (float)mantissa * pow2i((int)g - 11) : 0.0f;
        return sign ? -f : f;
    }
};

template <int D, int MODE, bool HAD>
SA_D void read_keys(const uint8_t* half, const CacheArgs& a, int t, uint4* row) {
    KeyReader<D, MODE> key(half, a, t);
    if constexpr (HAD) {
        float x[D];
#pragma unroll
        for (int c = 0; c < D / 8; ++c) {
            float y[8];
            key.get(c, y);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[8 * c + i] = y[i];
        }
        rotate_back<D>(x);
#pragma unroll
        for (int c = 0; c < D / 8; ++c)
            row[c ^ (t & 7)] = make_uint4(half2_bits(x[8 * c], x[8 * c + 1]), half2_bits(x[8 * c + 2], x[8 * c + 3]),
                                          half2_bits(x[8 * c + 4], x[8 * c + 5]), half2_bits(x[8 * c + 6], x[8 * c + 7]));
    } else {
#pragma unroll
        for (int c = 0; c < D / 8; ++c) {
            float x[8];
            key.get(c, x);
            row[c ^ (t & 7)] = make_uint4(half2_bits(x[0], x[1]), half2_bits(x[2], x[3]), half2_bits(x[4], x[5]), half2_bits(x[6], x[7]));
        }
    }
}
template <int D, int MODE>
SA_D void read_values(const uint8_t* half, const CacheArgs& a, int t, uint4* row) {
    const uint8_t* v = half + a.v_off;
    if constexpr (MODE == 16) {
#pragma unroll
        for (int c = 0; c < D / 8; ++c) row[c ^ (t & 7)] = load_16_bytes(v + ((size_t)c * kTileTokens + t) * 16);
    } else {
        // times 2^-g in two exact steps: the first keeps clear of the subnormal numbers, the second rounds where the value is one
        const int g = (int)(int8_t)half[a.meta_off + t * 4 + 2], g1 = max(-10, min(g, 12));
        const uint32_t f1 = half2_bits(pow2i(-g1), pow2i(-g1)), f2 = half2_bits(pow2i(max(g1 - g, -40)), pow2i(max(g1 - g, -40)));
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
            const uint4 in = load_16_bytes(v + ((size_t)k * kTileTokens + t) * 16);
            const uint32_t w[4] = {in.x, in.y, in.z, in.w};
            uint32_t h[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t even = int8_to_half2<false>(w[i]), odd = int8_to_half2<true>(w[i]);
                h[2 * i] = mul_half2(mul_half2(__byte_perm(even, odd, 0x5410), f1), f2);
                h[2 * i + 1] = mul_half2(mul_half2(__byte_perm(even, odd, 0x7632), f1), f2);
            }
            row[(2 * k) ^ (t & 7)] = make_uint4(h[0], h[1], h[2], h[3]);
            row[(2 * k + 1) ^ (t & 7)] = make_uint4(h[4], h[5], h[6], h[7]);
        }
    }
}

template <int D, int MODE, bool HAD>
__global__ void __launch_bounds__(128, HAD || (MODE == 33 && D == 128) ? 0 : D == 64 ? 9 : 8) read_kernel(CacheArgs a, uint16_t* Kout, uint16_t* Vout, const __grid_constant__ ReadSeqs seqs) {
    const int lane = threadIdx.x & 31;
    const int parts = Kout && Vout ? 2 : 1;
    const uint32_t unit = blockIdx.x * 4 + (threadIdx.x >> 5), each = (uint32_t)(parts * a.Hkv);      // (tile, head, keys or values)
    const int tile = (int)(unit / each), rest = (int)(unit % each);
    const int head = rest / parts;
    const bool values = parts == 2 ? rest & 1 : Kout == nullptr;
    if (tile >= seqs.tiles[seqs.n]) return;
    int i = 0;                                                                    // the sequence: the last one that starts at or before the tile
    for (int j0 = 0; j0 < seqs.n; j0 += 32) {
        const int j = j0 + lane;
        i += __popc(__ballot_sync(0xffffffffu, j < seqs.n && seqs.tiles[j + 1] <= tile));
    }
    const int start = seqs.start[i], t0 = ((start >> 5) + tile - seqs.tiles[i]) * kTileTokens;        // first token of the half page
    const int first = max(start - t0, 0), end = min(start + seqs.len[i] - t0, kTileTokens);            // of its tokens: those asked for
    pdl_wait();                                                                   // earlier kernels may still write this cache
    const uint8_t* block = page_block(a, seqs.b0 + i, t0 / kPageTokens, head);
    constexpr int C = D / 8, R = 32 / C;
    const int64_t row0 = seqs.row0[i] + t0 - start;                               // (of the half page's first token)
    if constexpr (MODE == 33)                                                     // 4 bits: a lane has a block of 16 channels (sa_fp4.cuh)
        if (block) {
            fp4_read<D, HAD>(block + (size_t)((t0 % kPageTokens) >> 5) * (a.page_bytes >> 1), a.v_off, values,
                             (values ? Vout : Kout) + (row0 * a.Hkv + head) * D, (int64_t)a.Hkv * D, first, end, lane);
            return;
        }
    __shared__ uint4 buffers[4][MODE == 33 ? 1 : 32 * C];
    uint4* rows = buffers[threadIdx.x >> 5];
    if (MODE != 33 && block) {
        const uint8_t* half = block + (size_t)((t0 % kPageTokens) >> 5) * (a.page_bytes >> 1);
        if (values) read_values<D, MODE>(half, a, lane, rows + lane * C);
        else read_keys<D, MODE, HAD>(half, a, lane, rows + lane * C);
    }
    __syncwarp();
    const int ch = lane % C;
    uint4* out = reinterpret_cast<uint4*>(values ? Vout : Kout) + head * C + ch;
#pragma unroll
    for (int k = 0; k < C; ++k) {
        const int row = k * R + lane / C;
        if (row >= first && row < end) out[(row0 + row) * (a.Hkv * C)] = block ? rows[row * C + (ch ^ (row & 7))] : make_uint4(0u, 0u, 0u, 0u);
    }
}

// Half pages that tokens start .. start + n - 1 lie in (their end may be 2^31 - 1: no sums in 32 bits).
static int64_t half_pages(int64_t start, int64_t n) { return n ? (start + n + kTileTokens - 1) / kTileTokens - start / kTileTokens : 0; }

template <int D, int MODE, bool HAD>
static void launch_read(const CacheArgs& a, uint16_t* K, uint16_t* V, const ReadSeqs& seqs, unsigned grid, cudaStream_t s) {
    (void)launch_pdl(read_kernel<D, MODE, HAD>, dim3(grid), dim3(128), 0, s, a, K, V, seqs);
}
template <int D>
static void launch_read(int mode, const CacheArgs& a, uint16_t* K, uint16_t* V, const ReadSeqs& seqs, unsigned grid, cudaStream_t s) {
#define CALL(M)                                                              \
    case M:                                                                  \
        if (M != 16 && a.hadamard) launch_read<D, M, M != 16>(a, K, V, seqs, grid, s); \
        else launch_read<D, M, false>(a, K, V, seqs, grid, s);               \
        break
    switch (mode) {
        CALL(4);
        CALL(8);
        CALL(9);
        CALL(10);
        CALL(16);
        CALL(32);
        CALL(33);
    }
#undef CALL
}

}  // namespace sa

using namespace sa;

extern "C" sa_status sa_read_kv(const sa_config* cfg, const sa_cache* cache, const int64_t* starts_host, const int64_t* cu_lens_host,
                                uint16_t* K, uint16_t* V, sa_stream stream) {
    Plan p;
    sa_status st = make_plan(cfg, &p);
    if (st != SA_OK) return st;
    CacheArgs a;
    st = check_cache(p, cache, &a);
    if (st != SA_OK) return st;
    if (!cu_lens_host) return SA_ERR_INVALID_ARG;
    if (!aligned(K, 16) || !aligned(V, 16)) return SA_ERR_ALIGNMENT;
    int64_t most = (int64_t)a.max_pages * kPageTokens, tiles = 0;
    if (most > 0x7fffffffLL) most = 0x7fffffffLL;                                 // (lengths are 32-bit numbers)
    for (int b = 0; b < a.batch; ++b) {
        const int64_t n = cu_lens_host[b + 1] - cu_lens_host[b], start = starts_host ? starts_host[b] : 0;
        if (n < 0 || cu_lens_host[b] < 0 || start < 0) return SA_ERR_INVALID_ARG;
        if (start > most || n > most - start) return SA_ERR_CAPACITY;
        tiles += half_pages(start, n);
    }
    if (tiles == 0) return SA_OK;                                                 // (a tensor without elements has no address)
    if (!K && !V) return SA_ERR_INVALID_ARG;
    const int parts = K && V ? 2 : 1;
    if (tiles * parts * a.Hkv > 0xfffffff0LL || tiles > 0x7fffffffLL) return SA_ERR_CAPACITY;      // (of all launches together: none is made before the last check)
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    // the byte container holds the codes of any number of mantissa bits alike
    const int mode = p.fp16 ? 16 : p.fp4 ? 33 : p.int8 ? 32 : p.nibble ? 8 + p.k : 4;
    for (int b0 = 0; b0 < a.batch; b0 += kReadBatch) {
        ReadSeqs seqs{};
        seqs.b0 = b0;
        seqs.n = a.batch - b0 < kReadBatch ? a.batch - b0 : kReadBatch;
        for (int i = 0; i < seqs.n; ++i) {
            seqs.row0[i] = cu_lens_host[b0 + i];
            seqs.start[i] = starts_host ? (int)starts_host[b0 + i] : 0;
            seqs.len[i] = (int)(cu_lens_host[b0 + i + 1] - cu_lens_host[b0 + i]);
            seqs.tiles[i + 1] = seqs.tiles[i] + (int)half_pages(seqs.start[i], seqs.len[i]);
        }
        const int64_t units = (int64_t)seqs.tiles[seqs.n] * parts * a.Hkv;
        if (units == 0) continue;
        const unsigned grid = (unsigned)((units + 3) / 4);
        if (p.d == 64) launch_read<64>(mode, a, K, V, seqs, grid, s);
        else launch_read<128>(mode, a, K, V, seqs, grid, s);
        if (cudaGetLastError() != cudaSuccess) return SA_ERR_CUDA;
    }
    return SA_OK;
}
