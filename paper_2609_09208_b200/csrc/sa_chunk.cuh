// Attention of several new tokens per sequence over the paged cache (sa_chunk_attention): the kernel.
//
// O = softmax(Q K^T / sqrt(d)) V for the last n tokens of a sequence, over every kind of cache, each token over what is not behind it, or over a
// window and the first few tokens.  The rows of a product are (token, query head of the KV head's group) pairs, so that a group's heads share a tile of keys.
//
// A block (one per SM) walks through pieces: 128 or 256 rows of one (sequence, KV head) and a stretch of tiles of 128 keys.  Its warps:
//   loader     copies the pages' records as they are into a ring in shared memory (bulk copies);
//   4 warps    turn the records of a tile into operands, 16 bits a number: a key's code (PoT: bfloat16, INT8, 4 bits, binary16: binary16) without its
//              scale, which the softmax applies in FP32 to the sums, and values as the binary16 numbers that the codes stand for: both exact, as the
//              decode kernels' operands are;
//   1 thread   issues the products (tcgen05): S = Q K^T into tensor memory, O += P V with the weights P read from there;
//   2 x 4 warps, a row a thread: the online softmax.  The weights take the place of the scores that they come from.
// Two streams of products take turns, so that the tensor core works on one while the softmax works on the other: two tiles of 128 rows
// against the same keys; or, where a sequence has no more than 128 rows (SPLIT), the same rows against every other tile of keys.  Of few rows a tile of
// 128 is filled up with copies, each for a part of the tile's keys (a thread then has 32 or 64 scores of a tile, not 128); the parts' sums meet at the end.
//
// Statistics and sums are FP32.  A weight is 2^(z - M + 7), z the logit in the log2 domain and M a reference that follows the row's maximum once that has grown by
// 8 (the sums are rescaled then): weights stay below 2^15, and what is 2^-21 of the largest keeps its 11 bits as a binary16 number.  That rounding, 2^-12 on
// average and independent from key to key, costs an output no more than its own rounding to binary16 does.
//
// Work is dealt on the device, as only that knows the lengths: units (KV head, sequence, row tile) in order, each with its tiles and a fixed cost, are cut into
// equal stretches, one a block.  A unit that a cut goes through leaves partial sums in the workspace, two places a block, for chunk_merge_kernel.
#pragma once
#include <cuda_bf16.h>

#include "sa_cache_write.cuh"
#include "sa_common.cuh"
#include "sa_fp4.cuh"
#include "sa_score_mma.cuh"
#include "sa_stage.cuh"
#include "sa_tcgen05.cuh"

namespace sa {

constexpr int kChunkBatch = 128;          // sequences per launch
constexpr int kChunkThreads = 448;        // 2 x 4 warps of softmax, 4 of operands, products, loader
constexpr int kChunkTile = 128;           // keys
constexpr int kChunkUnitCost = 4;         // what a unit costs beside its tiles, in tiles
constexpr int kChunkPlanBytes = 16384;    // of the workspace, ahead of the partial sums: a ChunkCut a block
constexpr int kChunkBlocksMost = kChunkPlanBytes / 16;
SA_HD constexpr int chunk_rows(bool split) { return split ? 128 : 256; }
SA_HD constexpr size_t chunk_slot_floats(int d, bool split) { return (size_t)chunk_rows(split) * (d + 2); }

struct ChunkSeqs {
    int n;                                // sequences of this launch
    int b[kChunkBatch];                   // each: its number in the cache
    int tokens[kChunkBatch];              // new tokens, and their first row in Q and O
    int64_t row0[kChunkBatch];
    int tiles[kChunkBatch + 1];           // row tiles ahead of it
};
struct ChunkArgs {
    CacheArgs c;
    const uint16_t* Q;
    void* O;
    uint8_t* workspace;
    int Hq, G, window, sinks;
    int copies;                           // SPLIT: 1, 2 or 4 copies of the rows in a tile
    int bf16;                             // type of O
    float factor;                         // log2(e) / sqrt(d) and the unit of the operands
    ChunkSeqs s;
};
// A unit that the cut behind a block goes through and that starts in it: its parts are the block's second place and the first places of the blocks up to `last`.
struct ChunkCut {
    int head, tile, last, there;
};

// Key tiles that the rows of a row tile need, in the order in which they are taken: those of the first tokens, then those of the window.
struct ChunkUnit {
    int seq, row0, rows;                  // in the launch; rows of the sequence's (token, head of the group) pairs
    int first, last;                      // positions of the first and the last row's token
    int lo, hi;                           // keys lo .. hi - 1, and below sinks
    int sink_tiles, window_tile, count;
    SA_D int tile(int i) const { return i < sink_tiles ? i : window_tile + i - sink_tiles; }
};
SA_D ChunkUnit chunk_unit(const ChunkArgs& a, const int* lens, int flat, int per_tile) {
    int lo = 0, hi = a.s.n;               // the sequence: the last one whose row tiles start at or before this one
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (a.s.tiles[mid] <= flat) lo = mid;
        else hi = mid;
    }
    ChunkUnit u;
    u.seq = lo;
    u.row0 = (flat - a.s.tiles[lo]) * per_tile;
    u.rows = min(per_tile, a.s.tokens[lo] * a.G - u.row0);
    const int before = lens[lo] - a.s.tokens[lo];
    u.first = before + u.row0 / a.G;
    u.last = before + (u.row0 + u.rows - 1) / a.G;
    const int most = a.c.max_pages > 0x7fffffff / kPageTokens ? 0x7fffffff : a.c.max_pages * kPageTokens;
    u.hi = min(u.last, most - 1) + 1;
    u.lo = a.window && u.first >= a.window ? u.first - a.window + 1 : 0;
    u.sink_tiles = u.window_tile = u.count = 0;
    if (u.hi > 0) {
        const int end = (u.hi - 1) / kChunkTile + 1;
        u.window_tile = min(u.lo / kChunkTile, end);
        u.sink_tiles = u.lo && a.sinks ? min((min(a.sinks, u.hi) - 1) / kChunkTile + 1, u.window_tile) : 0;
        u.count = u.sink_tiles + end - u.window_tile;
    }
    return u;
}

// The pieces of a block, in order; every warp walks through them by itself.
struct ChunkPiece {
    ChunkUnit u;
    int head, flat, begin, end;           // tiles begin .. end - 1 of the unit's
    SA_D bool whole() const { return begin == 0 && end == u.count; }
};
struct ChunkWalk {
    int head, flat, skip;                 // the unit, and how far into it (its fixed cost included) the stretch starts
    long long left;                       // of the stretch
    SA_D bool next(const ChunkArgs& a, const int* lens, int per_tile, ChunkPiece& p) {
        while (left > 0) {
            p.u = chunk_unit(a, lens, flat, per_tile);
            p.head = head;
            p.flat = flat;
            const int cost = kChunkUnitCost + p.u.count, from = skip;
            const int to = left < cost - from ? from + (int)left : cost;
            left -= to - from;
            skip = 0;
            if (++flat == a.s.tiles[a.s.n]) flat = 0, ++head;
            p.begin = max(from - kChunkUnitCost, 0);
            p.end = max(to - kChunkUnitCost, 0);
            if (p.end > p.begin || (p.u.count == 0 && from == 0)) return true;
        }
        return false;
    }
};

// Shared memory of a block.
template <int D, int FMT>
struct ChunkShape {
    static constexpr int kHalf = FMT == FMT_FP16 ? half_block_bytes_fp16(D) : FMT == FMT_FP4 ? half_block_bytes_fp4(D)
                                 : half_block_bytes(D, FMT == FMT_PLANAR1 ? 1 : FMT == FMT_PLANAR2 ? 2 : FMT == FMT_INT8 ? 8 : 0, FMT == FMT_NIBBLE || FMT == FMT_PLANAR1 || FMT == FMT_PLANAR2);
    static constexpr int kRaw = 4 * kHalf;                            // records of a tile
    static constexpr int kOperand = D / 64 * 16384;                   // 128 rows
    static constexpr int kBuffers = D == 64 ? 2 : 1;                  // of operands
    static constexpr int kFixed = (2 + 2 * kBuffers) * kOperand + 8192;
    static constexpr int kFit = (227 * 1024 - 1024 - kFixed) / kRaw;
    static constexpr int kStages = kFit > 4 ? 4 : kFit;
    static constexpr int kBytes = 1024 + kFixed + kStages * kRaw;     // (1024: to align)
    static constexpr int kV = (FMT == FMT_FP16) ? 64 * D : FMT == FMT_FP4 ? 18 * D : kHalf - 32 * D;      // offset of the values in a half
    static constexpr int kMeta = FMT == FMT_FP4 ? 16 * D : kV - 128;
    static constexpr bool kScaled = FMT != FMT_FP16 && FMT != FMT_FP4;                                  // keys have a scale of their own
    static constexpr bool kBf16 = kScaled && FMT != FMT_INT8;                                           // type of keys and queries
    static_assert(kStages >= 1, "a tile's records have to fit");
};
struct ChunkShared {                      // behind the rings
    float scale[4][kChunkTile];           // of the keys of four tiles
    float m[256], l[256];
    uint32_t pages[4];                    // which of a tile's pages there are
    uint32_t raw_info[4];
    unsigned long long raw_full[4], raw_empty[4], k_full[2], k_empty[2], v_full[2], v_empty[2], q_full[2], s_full[2], p_full[2], o_full[2], done;
    int lens[kChunkBatch];
    uint32_t tmem;
    int start_head, start_flat, start_skip;
    long long sums[16];
};
static_assert(sizeof(ChunkShared) <= 8192, "room behind the rings");

// A wait that ends: where the limit is reached, nothing is waited for any more and the outputs become NaN.
struct ChunkWait {
    bool lost = false;
    SA_D void one(const unsigned long long& bar, uint32_t parity) {
        if (!lost) lost = !mbar_wait_bounded(smem_addr(&bar), parity);
    }
    SA_D void operator()(const unsigned long long& bar, uint32_t parity) {      // a whole warp
        one(bar, parity);
        __syncwarp();
    }
};

SA_D uint32_t swizzled(int row, int piece) { return (uint32_t)(row * 128 + ((piece ^ (row & 7)) << 4)); }
SA_D void sts_16(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
// Operand row `row`, channels 8 c .. 8 c + 7.
SA_D void put_operand(uint32_t operand, int row, int c, uint32_t a, uint32_t b, uint32_t x, uint32_t y) {
    sts_16(operand + (c >> 3) * 16384 + swizzled(row, c & 7), a, b, x, y);
}
// Codes of a word of nibbles (sign << 3 | g), two at a time (channels 2 i, 2 i + 1 of byte i), as bfloat16 numbers, 2^-120 of the codes'.
SA_D uint32_t nibbles_to_bf16(uint32_t w, int i) {
    const uint32_t h = ((w >> (8 * i)) & 0xffu) * 0x1001u;
    return ((h << 7) & 0x03800380u) | ((h << 12) & 0x80008000u);
}
// Bits 2 i, 2 i + 1 of a plane's byte, at bit AT of two 16-bit numbers.
template <int AT>
SA_D uint32_t plane_pair(uint32_t p, int i) {
    const uint32_t q = (p >> (2 * i)) & 3u;
    return ((q | q << 15) & 0x00010001u) << AT;
}

// The key of one token (t of a half) as a row of the operand.
template <int D, int FMT>
SA_D void chunk_key(const uint8_t* half, int t, uint32_t operand, int row) {
    const uint4* chunk = reinterpret_cast<const uint4*>(half) + t;                      // + 32 k: chunk k
    if constexpr (FMT == FMT_FP16) {
#pragma unroll
        for (int c = 0; c < D / 8; ++c) {
            const uint4 w = chunk[32 * c];
            put_operand(operand, row, c, w.x, w.y, w.z, w.w);
        }
    } else if constexpr (FMT == FMT_FP4) {
#pragma unroll
        for (int k = 0; k < D / 32; ++k) {
            const uint4 v = chunk[32 * k];
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t b = half[16 * D + k / 2 * 128 + i * 32 + t % 8 * 4 + t / 8], s = b << 7 | b << 23;
                uint32_t h[4];
                fp4_to_half2(w[i], h);
                put_operand(operand, row, 8 * (k / 2) + 2 * i + k % 2, mul_half2(h[0], s), mul_half2(h[1], s), mul_half2(h[2], s), mul_half2(h[3], s));
            }
        }
    } else if constexpr (FMT == FMT_BYTE || FMT == FMT_INT8) {
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
            const uint4 v = chunk[32 * k];
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
            uint32_t h[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (FMT == FMT_BYTE) {
                    h[2 * i] = byte_codes_to_bf16<0>(w[i], 1u);
                    h[2 * i + 1] = byte_codes_to_bf16<2>(w[i], 1u);
                } else {
                    const uint32_t even = int8_to_half2<false>(w[i]), odd = int8_to_half2<true>(w[i]);
                    h[2 * i] = __byte_perm(even, odd, 0x5410);
                    h[2 * i + 1] = __byte_perm(even, odd, 0x7632);
                }
            }
            put_operand(operand, row, 2 * k, h[0], h[1], h[2], h[3]);
            put_operand(operand, row, 2 * k + 1, h[4], h[5], h[6], h[7]);
        }
    } else {
        constexpr int K = FMT == FMT_PLANAR1 ? 1 : FMT == FMT_PLANAR2 ? 2 : 0;
#pragma unroll
        for (int k = 0; k < D / 32; ++k) {
            const uint4 v = chunk[32 * k];
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
            uint32_t plane[K ? K : 1] = {};
#pragma unroll
            for (int bit = 0; bit < K; ++bit) plane[bit] = *reinterpret_cast<const uint32_t*>(half + 16 * D + (bit * kTileTokens + t) * (D / 8) + 4 * k);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t h[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    h[i] = nibbles_to_bf16(w[c], i);
                    if constexpr (K == 1) h[i] |= plane_pair<6>(plane[0] >> (8 * c), i);
                    if constexpr (K == 2) h[i] |= plane_pair<5>(plane[0] >> (8 * c), i) | plane_pair<6>(plane[1] >> (8 * c), i);
                }
                put_operand(operand, row, 4 * k + c, h[0], h[1], h[2], h[3]);
            }
        }
    }
}
// Its value.
template <int D, int FMT>
SA_D void chunk_value(const uint8_t* half, int t, uint32_t operand, int row) {
    using S = ChunkShape<D, FMT>;
    const uint8_t* v = half + S::kV;
    if constexpr (FMT == FMT_FP16) {
#pragma unroll
        for (int c = 0; c < D / 8; ++c) {
            const uint4 w = reinterpret_cast<const uint4*>(v)[32 * c + t];
            put_operand(operand, row, c, w.x, w.y, w.z, w.w);
        }
    } else if constexpr (FMT == FMT_FP4) {
        const uint8_t* at = v + t % 8 / 2 * 16 + t / 16 * 4 + t / 8 % 2 * 2;
        const uint8_t* scales = v + 16 * D + t % 8 / 2 * 16 + t / 16 * 4 + t % 2 * 2 + t / 8 % 2;
        const int shift = 4 * (t & 1);
#pragma unroll
        for (int blk = 0; blk < D / 16; ++blk) {
            uint32_t x[8], w[2], h[4];                                                  // x[e]: channels e, e + 8 of the block
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = (uint32_t)*reinterpret_cast<const uint16_t*>(at + blk / 2 * 512 + e * 64 + blk % 2 * 8) >> shift & 0x0f0fu;
#pragma unroll
            for (int e = 0; e < 8; e += 2) x[e] |= x[e + 1] << 4;
            const uint32_t lo = x[0] | x[2] << 16, hi = x[4] | x[6] << 16;
            w[0] = __byte_perm(lo, hi, 0x6420);
            w[1] = __byte_perm(lo, hi, 0x7531);
            const uint32_t b = scales[blk / 2 * 64 + blk % 2 * 8], s = b << 7 | b << 23;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                fp4_to_half2(w[i], h);
                put_operand(operand, row, 2 * blk + i, mul_half2(h[0], s), mul_half2(h[1], s), mul_half2(h[2], s), mul_half2(h[3], s));
            }
        }
    } else {
        // times 2^-g in two exact steps: the first keeps clear of the subnormal numbers; the product is a number that binary16 has, as the value that was
        // rounded was one, but for 65536, which becomes the largest
        const int g = (int)(int8_t)half[S::kMeta + t * 4 + 2], g1 = max(-9, min(g, 12));
        const __half f1h = __float2half_rn(pow2i(-g1)), f2h = __float2half_rn(pow2i(max(g1 - g, -40)));
        const uint32_t f1 = (uint32_t)__half_as_ushort(f1h) * 0x10001u, f2 = (uint32_t)__half_as_ushort(f2h) * 0x10001u;
        const bool twice = __any_sync(0xffffffffu, g != g1);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
            const uint4 in = reinterpret_cast<const uint4*>(v)[32 * k + t];
            const uint32_t w[4] = {in.x, in.y, in.z, in.w};
            uint32_t h[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t even = int8_to_half2<false>(w[i]), odd = int8_to_half2<true>(w[i]);
                h[2 * i] = mul_half2(__byte_perm(even, odd, 0x5410), f1);
                h[2 * i + 1] = mul_half2(__byte_perm(even, odd, 0x7632), f1);
            }
            if (twice)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    h[i] = mul_half2(h[i], f2);
                    asm("{.reg .b32 m; mov.b32 m, 0x7bff7bff; min.f16x2 %0, %0, m; neg.f16x2 m, m; max.f16x2 %0, %0, m;}" : "+r"(h[i]));
                }
            put_operand(operand, row, 2 * k, h[0], h[1], h[2], h[3]);
            put_operand(operand, row, 2 * k + 1, h[4], h[5], h[6], h[7]);
        }
    }
}

// The 32 queries of a warp as rows of the operand, D / 16 lanes a row; returns the factor of the lane's own row.  row_of(r): row r's binary16 numbers, or null.
template <int D, int FMT, typename RowOf>
SA_D float chunk_queries(const ChunkArgs& a, uint32_t operand, int lane, int first_row, RowOf row_of) {
    using S = ChunkShape<D, FMT>;
    constexpr int LPV = D / 16, RPW = 32 / LPV, STEPS = 32 / RPW;
    const Fp4Half<D> f(lane, 0);
    uint32_t x[STEPS][8];
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const uint16_t* p = row_of(i * RPW + lane / LPV);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] = 0u;
        if (p) load_32_bytes(p + 16 * f.blk, (reinterpret_cast<uintptr_t>(a.Q) & 31) == 0, x[i]);
    }
    float mine = a.factor;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        if (a.c.hadamard) f.rotate(x[i]);
        if constexpr (S::kScaled) {                                                     // as quantise_query_vec: 127 steps of the largest magnitude
            uint32_t top = x[i][0] & 0x7fff7fffu;
#pragma unroll
            for (int e = 1; e < 8; ++e) top = __vmaxu2(top, x[i][e] & 0x7fff7fffu);
            top = max(top & 0xffffu, top >> 16);
#pragma unroll
            for (int o = 1; o < LPV; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
            const float amax = half_bits_to_float(top), inv = top ? __fdiv_rn(127.0f, amax) : 0.0f, delta = __fdiv_rn(amax, 127.0f);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&x[i][e]));
                const float lo = fminf(fmaxf(rintf(__fmul_rn(v.x, inv)), -127.0f), 127.0f), hi = fminf(fmaxf(rintf(__fmul_rn(v.y, inv)), -127.0f), 127.0f);
                if constexpr (S::kBf16) {
                    const __nv_bfloat162 h = __floats2bfloat162_rn(lo * 0x1p112f, hi * 0x1p112f);      // (the keys' numbers are 2^-120 of the codes')
                    x[i][e] = *reinterpret_cast<const uint32_t*>(&h);
                } else {
                    const __half2 h = __floats2half2_rn(lo, hi);
                    x[i][e] = *reinterpret_cast<const uint32_t*>(&h);
                }
            }
            const float d = __shfl_sync(0xffffffffu, top ? delta : 1.0f, (lane % RPW) * LPV);      // (a query of zeros: any factor but zero)
            if (lane / RPW == i) mine = d * a.factor;
        }
        const int row = first_row + i * RPW + lane / LPV;
        put_operand(operand, row, 2 * f.blk, x[i][0], x[i][1], x[i][2], x[i][3]);
        put_operand(operand, row, 2 * f.blk + 1, x[i][4], x[i][5], x[i][6], x[i][7]);
    }
    return mine;
}

SA_D uint32_t half2_of(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// Channels of an output row, two a register.
SA_D uint32_t chunk_out(float a, float b, int bf16) {
    if (!bf16) return half2_of(a, b);
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
SA_D uint32_t bits_below(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }
SA_D void chunk_sync(int barrier, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(threads) : "memory"); }

// Row r of a unit: its number in Q and O.
SA_D int64_t chunk_row(const ChunkArgs& a, const ChunkUnit& u, int head, int r) {
    const int at = u.row0 + r, token = at / a.G;
    return (a.s.row0[u.seq] + token) * a.Hq + head * a.G + (at - token * a.G);
}

template <int D, int FMT, bool SPLIT>
__global__ void __launch_bounds__(kChunkThreads, 1) chunk_kernel(const __grid_constant__ ChunkArgs a) {
    using S = ChunkShape<D, FMT>;
    constexpr int kPerTile = chunk_rows(SPLIT), NB = S::kBuffers;
    extern __shared__ uint8_t dynamic[];
    const uint32_t base = (smem_addr(dynamic) + 1023u) & ~1023u;
    uint8_t* const rings = dynamic + (base - smem_addr(dynamic));
    const uint32_t q_at = base, k_at = q_at + 2 * S::kOperand, v_at = k_at + NB * S::kOperand;
    uint8_t* const raw = rings + (2 + 2 * NB) * S::kOperand;
    ChunkShared& sh = *reinterpret_cast<ChunkShared*>(raw + S::kStages * S::kRaw);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int per_tile = SPLIT ? kPerTile / a.copies : kPerTile;

    if (tid == 0) {
        for (int i = 0; i < 4; ++i) {
            mbar_init(smem_addr(&sh.raw_full[i]), 1);
            mbar_init(smem_addr(&sh.raw_empty[i]), 4);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_addr(&sh.k_full[i]), 4);
            mbar_init(smem_addr(&sh.v_full[i]), 4);
            mbar_init(smem_addr(&sh.k_empty[i]), 1);
            mbar_init(smem_addr(&sh.v_empty[i]), 1);
            mbar_init(smem_addr(&sh.q_full[i]), 4);
            mbar_init(smem_addr(&sh.s_full[i]), 2);                    // (the products' arrival, and the issuing thread's own, which hands on what it has seen)
            mbar_init(smem_addr(&sh.p_full[i]), 4);
            mbar_init(smem_addr(&sh.o_full[i]), 1);
        }
        mbar_init(smem_addr(&sh.done), 1);
        fence_mbar_init();
    }
    pdl_wait();
    pdl_launch_dependents();

    // ---- the deal
    const int n_flat = a.s.tiles[a.s.n];
    if (tid < a.s.n) sh.lens[tid] = max(a.c.seq_lens[a.s.b[tid]], 0);
    __syncthreads();
    const int each = (n_flat + kChunkThreads - 1) / kChunkThreads, mine0 = min(tid * each, n_flat), mine1 = min(mine0 + each, n_flat);
    long long cost = 0;
    for (int i = mine0; i < mine1; ++i) cost += kChunkUnitCost + chunk_unit(a, sh.lens, i, per_tile).count;
    long long ahead = cost;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, ahead, o);
        if (lane >= o) ahead += x;
    }
    if (lane == 31) sh.sums[warp] = ahead;
    __syncthreads();
    long long sum = 0;
    ahead -= cost;
    for (int w = 0; w < kChunkThreads / 32; ++w) {
        if (w < warp) ahead += sh.sums[w];
        sum += sh.sums[w];
    }
    const long long total = sum * a.c.Hkv, blocks = min((long long)gridDim.x, total);
    ChunkCut* cuts = reinterpret_cast<ChunkCut*>(a.workspace);
    if (blockIdx.x >= blocks) {
        if (tid == 0) cuts[blockIdx.x].there = 0;
        return;
    }
    const long long x0 = total * blockIdx.x / blocks, x1 = total * (blockIdx.x + 1) / blocks;
    {
        const int head = (int)(x0 / sum);
        long long rest = x0 - head * sum - ahead;
        if (rest >= 0 && rest < cost) {                                // the unit at which the stretch starts is one of this thread's
            int i = mine0;
            for (;;) {
                const int c = kChunkUnitCost + chunk_unit(a, sh.lens, i, per_tile).count;
                if (rest < c) break;
                rest -= c;
                ++i;
            }
            sh.start_head = head;
            sh.start_flat = i;
            sh.start_skip = (int)rest;
        }
    }
    if (warp == 12) tmem_alloc(smem_addr(&sh.tmem));
    tcgen05_before_sync();
    __syncthreads();
    tcgen05_after_sync();
    const uint32_t tmem = sh.tmem;
    ChunkWalk walk{sh.start_head, sh.start_flat, sh.start_skip, x1 - x0};
    ChunkPiece p;
    ChunkWait wait;

    if (warp < 8) {
        // ---- softmax: a row a thread
        const int stream = warp >> 2, quarter = warp & 3, own = quarter * 32 + lane;
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16), s_col = lanes + stream * 128, o_col = lanes + 256 + stream * D;
        const uint32_t q_operand = q_at + stream * S::kOperand;
        const int copies = SPLIT ? a.copies : 1, rows_own = 128 / copies;
        const int row = SPLIT ? own % rows_own : stream * 128 + own;   // of the unit
        const int chunks = 4 / copies, chunk0 = SPLIT ? own / rows_own * chunks : 0;      // columns of 32 that this thread has
        uint32_t tiles_done = 0, pieces_done = 0, keys_done = 0;
        bool cut_here = false;
        while (walk.next(a, sh.lens, per_tile, p)) {
            const ChunkUnit& u = p.u;
            const bool there = row < u.rows;
            const int position = there ? u.first + (u.row0 + row) / a.G - u.row0 / a.G : -1;
            const int n = p.end - p.begin, mine = SPLIT ? (n + 1 - stream) / 2 : n;       // tiles of this stream
            float m = -1e30f, l = 0.0f, f = a.factor;
            if (n > 0) {
                const int first_row = SPLIT ? quarter * 32 : stream * 128 + quarter * 32;
                f = chunk_queries<D, FMT>(a, q_operand, lane, quarter * 32, [&](int r) -> const uint16_t* {
                    const int at = SPLIT ? (first_row + r) % rows_own : first_row + r;
                    return at < u.rows ? a.Q + chunk_row(a, u, p.head, at) * D : nullptr;
                });
                fence_proxy_async();
                tcgen05_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&sh.q_full[stream]));
            }
            // positions of the stream's first and last row: a tile that all of them see whole needs no masks
            const int row_lo = SPLIT ? 0 : min(stream * 128, u.rows - 1), row_hi = SPLIT ? u.rows - 1 : min(stream * 128 + 127, u.rows - 1);
            const int position_lo = u.first + (u.row0 + row_lo) / a.G - u.row0 / a.G, position_hi = u.first + (u.row0 + row_hi) / a.G - u.row0 / a.G;
            for (int i = 0; i < mine; ++i) {
                const int j = SPLIT ? 2 * i + stream : i, t0 = u.tile(p.begin + j) * kChunkTile, slot = (keys_done + j) & 3;
                wait(sh.s_full[stream], tiles_done & 1);
                ++tiles_done;
                tcgen05_after_sync();
                const uint32_t pages = sh.pages[slot];
                const float* scale = sh.scale[slot];
                const bool plain = pages == 3u && position_lo - t0 >= kChunkTile - 1 && (a.window == 0 || position_hi - t0 < a.window || t0 + kChunkTile <= a.sinks);
                const int hi = position - t0, lo = a.window && position >= 0 ? (int)max((long long)hi - a.window + 1, -0x40000000ll) : -0x40000000, sink = a.sinks - t0;
                auto scores = [&](int c, f32x2 (&y)[16]) {             // columns 32 c .. of the row, times the keys' scales; -inf where they are hidden
                    uint32_t x[32];
                    tmem_load(s_col + 32 * c, x);
                    tmem_loaded();
#pragma unroll
                    for (int e = 0; e < 16; ++e) y[e] = pack_f32x2(__uint_as_float(x[2 * e]), __uint_as_float(x[2 * e + 1]));
                    if constexpr (S::kScaled) {
#pragma unroll
                        for (int e = 0; e < 16; e += 2) {
                            const float4 s4 = *reinterpret_cast<const float4*>(scale + 32 * c + 2 * e);
                            y[e] = mul2(y[e], pack_f32x2(s4.x, s4.y));
                            y[e + 1] = mul2(y[e + 1], pack_f32x2(s4.z, s4.w));
                        }
                    }
                    if (!plain) {
                        const uint32_t seen = (pages >> (c >> 1) & 1u) ? bits_below(hi - 32 * c + 1) & (~bits_below(lo - 32 * c) | bits_below(sink - 32 * c)) : 0u;
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            float v, w;
                            unpack_f32x2(y[e], &v, &w);
                            y[e] = pack_f32x2(seen >> (2 * e) & 1u ? v : -INFINITY, seen >> (2 * e + 1) & 1u ? w : -INFINITY);
                        }
                    }
                };
                float top = -INFINITY;
#pragma unroll(SPLIT ? 1 : 4)
                for (int c = chunk0; c < chunk0 + chunks; ++c) {
                    f32x2 y[16];
                    scores(c, y);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        float v, w;
                        unpack_f32x2(y[e], &v, &w);
                        top = fmaxf(top, fmaxf(v, w));
                    }
                }
                const float z = top * f;
                const bool grown = z > m + 8.0f;
                if (__any_sync(0xffffffffu, grown)) {
                    const float r = grown ? ex2_approx(m - z) : 1.0f;
                    if (grown) m = z;
                    l *= r;
                    if (i > 0) {                                       // (the products of the tile before are done: the scores come behind them)
#pragma unroll 1
                        for (int c = 0; c < D; c += 32) {
                            uint32_t x[32];
                            tmem_load(o_col + c, x);
                            tmem_loaded();
#pragma unroll
                            for (int e = 0; e < 32; ++e) x[e] = __float_as_uint(__uint_as_float(x[e]) * r);
                            tmem_store(o_col + c, x);
                        }
                    }
                }
                const f32x2 f2 = pack_f32x2(f, f), m2 = pack_f32x2(7.0f - m, 7.0f - m);
                f32x2 l2 = pack_f32x2(0.0f, 0.0f);
#pragma unroll(SPLIT ? 1 : 4)
                for (int c = chunk0; c < chunk0 + chunks; ++c) {
                    f32x2 y[16];
                    scores(c, y);
                    uint32_t w[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        float u0, u1;
                        unpack_f32x2(ffma2(y[e], f2, m2), &u0, &u1);
                        u0 = ex2_approx(u0);
                        u1 = ex2_approx(u1);
                        l2 = add2(l2, pack_f32x2(u0, u1));
                        w[e] = half2_of(u0, u1);
                    }
                    tmem_store(s_col + 16 * c, w);
                }
                if constexpr (SPLIT) {
                    if (copies > 1) {
                        uint32_t zero[16] = {};
#pragma unroll 1
                        for (int c = 0; c < 4; ++c)
                            if (c < chunk0 || c >= chunk0 + chunks) tmem_store(s_col + 16 * c, zero);
                    }
                }
                float l0, l1;
                unpack_f32x2(l2, &l0, &l1);
                l += l0 + l1;
                tmem_stored();
                tcgen05_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&sh.p_full[stream]));
            }
            keys_done += n;
            if (n > 0) {
                wait(sh.o_full[stream], pieces_done & 1);
                ++pieces_done;
                tcgen05_after_sync();
            }
            // ---- the piece's sums
            const bool whole = p.whole();
            float* slot = nullptr;
            if (!whole) {
                slot = reinterpret_cast<float*>(a.workspace + kChunkPlanBytes) + (size_t)(2 * blockIdx.x + (p.begin == 0 ? 1 : 0)) * chunk_slot_floats(D, SPLIT);
                if (p.begin == 0) {
                    cut_here = true;
                    if (tid == 0) {
                        // the block that has the unit's last tile: the last one that starts at or before it
                        const long long x = x1 + p.u.count - p.end - 1;
                        cuts[blockIdx.x] = ChunkCut{p.head, p.flat, (int)(((x + 1) * blocks - 1) / total), 1};
                    }
                }
            }
            if constexpr (!SPLIT) {
                const float inv = wait.lost ? __int_as_float(0x7fc00000) : l > 0.0f ? __fdiv_rn(1.0f, l) : 0.0f;
                if (slot && there) {
                    slot[kPerTile * D + row] = m;
                    slot[kPerTile * (D + 1) + row] = wait.lost ? inv : l;
                }
                uint16_t* out = there ? static_cast<uint16_t*>(a.O) + chunk_row(a, u, p.head, row) * D : nullptr;
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    uint32_t x[32] = {};
                    if (mine > 0) {
                        tmem_load(o_col + c, x);
                        tmem_loaded();
                    }
                    if (there && slot) {
#pragma unroll
                        for (int e = 0; e < 32; e += 4) *reinterpret_cast<uint4*>(slot + (size_t)row * D + c + e) = make_uint4(x[e], x[e + 1], x[e + 2], x[e + 3]);
                    } else if (there) {
#pragma unroll
                        for (int e = 0; e < 32; e += 8) {
                            uint32_t w[4];
#pragma unroll
                            for (int k = 0; k < 4; ++k) w[k] = chunk_out(__uint_as_float(x[e + 2 * k]) * inv, __uint_as_float(x[e + 2 * k + 1]) * inv, a.bf16);
                            *reinterpret_cast<uint4*>(out + c + e) = make_uint4(w[0], w[1], w[2], w[3]);
                        }
                    }
                    __syncwarp();
                }
            } else {
                // 2 x copies parts of every row meet, 16 channels at a time, in the queries' place
                sh.m[tid] = m;
                sh.l[tid] = wait.lost ? __int_as_float(0x7fc00000) : l;
                chunk_sync(1, 256);
                __syncwarp();
                float most = -1e30f, all = 0.0f;
                for (int k = row; k < 256; k += rows_own) most = fmaxf(most, sh.m[k]);
                const float r = ex2_approx(m - most);
                float* exchange = reinterpret_cast<float*>(rings);
                constexpr int kPitch = 20;
                const int item_row = tid / (256 / rows_own), per_item = rows_own / 16, channel0 = tid % (256 / rows_own) * per_item;      // 2, 4 or 8 channels of a row
                {
                    float item_most = -1e30f;
                    for (int k = item_row; k < 256; k += rows_own) item_most = fmaxf(item_most, sh.m[k]);
                    for (int k = item_row; k < 256; k += rows_own) all += sh.l[k] * ex2_approx(sh.m[k] - item_most);
                    if (slot && channel0 == 0 && item_row < u.rows) {
                        slot[kPerTile * D + item_row] = item_most;
                        slot[kPerTile * (D + 1) + item_row] = all;
                    }
                }
                const float inv = all > 0.0f ? __fdiv_rn(1.0f, all) : all == 0.0f ? 0.0f : all;
                const bool item_there = item_row < u.rows;
                uint16_t* out = item_there ? static_cast<uint16_t*>(a.O) + chunk_row(a, u, p.head, item_row) * D : nullptr;
#pragma unroll 1
                for (int c = 0; c < D; c += 16) {
                    uint32_t x[16] = {};
                    if (mine > 0) {
                        tmem_load(o_col + c, x);
                        tmem_loaded();
                    }
#pragma unroll
                    for (int e = 0; e < 16; e += 4)
                        *reinterpret_cast<float4*>(exchange + tid * kPitch + e) =
                            make_float4(__uint_as_float(x[e]) * r, __uint_as_float(x[e + 1]) * r, __uint_as_float(x[e + 2]) * r, __uint_as_float(x[e + 3]) * r);
                    chunk_sync(1, 256);
                    if (item_there)
                        for (int e = 0; e < per_item; e += 2) {
                            float2 v = make_float2(0.0f, 0.0f);
                            for (int k = item_row; k < 256; k += rows_own) {
                                const float2 w = *reinterpret_cast<const float2*>(exchange + k * kPitch + channel0 + e);
                                v.x += w.x;
                                v.y += w.y;
                            }
                            if (slot) *reinterpret_cast<float2*>(slot + (size_t)item_row * D + c + channel0 + e) = v;
                            else *reinterpret_cast<uint32_t*>(out + c + channel0 + e) = chunk_out(v.x * inv, v.y * inv, a.bf16);
                        }
                    __syncwarp();
                    chunk_sync(1, 256);
                }
            }
            tcgen05_before_sync();
        }
        if (tid == 0 && !cut_here) cuts[blockIdx.x].there = 0;
    } else if (warp < 12) {
        // ---- operands: a key a thread
        const int part = warp - 8, row = part * 32 + lane;             // half page of the tile
        uint32_t keys_done = 0;
        while (walk.next(a, sh.lens, per_tile, p))
            for (int j = p.begin; j < p.end; ++j, ++keys_done) {
                const int stage = keys_done % S::kStages, buffer = keys_done % NB, slot = keys_done & 3;
                const uint32_t turn = keys_done / NB & 1;
                const int key = p.u.tile(j) * kChunkTile + row;
                wait(sh.raw_full[stage], keys_done / S::kStages & 1);
                const uint8_t* half = raw + stage * S::kRaw + part * S::kHalf;
                const uint32_t pages = sh.raw_info[stage];
                // what no row sees is zero: it may hold anything, and a weight of zero times that is not zero
                const bool seen = (pages >> (part >> 1) & 1u) && key < p.u.hi && (key >= p.u.lo || key < a.sinks);
                wait(sh.k_empty[buffer], turn ^ 1);
                const uint32_t k_operand = k_at + buffer * S::kOperand, v_operand = v_at + buffer * S::kOperand;
                if (seen) chunk_key<D, FMT>(half, lane, k_operand, row);
                else
#pragma unroll
                    for (int c = 0; c < D / 8; ++c) put_operand(k_operand, row, c, 0u, 0u, 0u, 0u);
                if constexpr (S::kScaled) sh.scale[slot][row] = seen ? half_bits_to_float(*reinterpret_cast<const uint16_t*>(half + S::kMeta + lane * 4)) : 0.0f;
                if (row == 0) sh.pages[slot] = pages;
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&sh.k_full[buffer]));
                wait(sh.v_empty[buffer], turn ^ 1);
                chunk_value<D, FMT>(half, lane, v_operand, row);
                if (!seen)
#pragma unroll
                    for (int c = 0; c < D / 8; ++c) put_operand(v_operand, row, c, 0u, 0u, 0u, 0u);
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(smem_addr(&sh.v_full[buffer]));
                    mbar_arrive(smem_addr(&sh.raw_empty[stage]));
                }
            }
    } else if (warp == 12) {
        // ---- products
        if (lane == 0) {
            constexpr uint32_t kScores = mma_form(kChunkTile, S::kBf16, false), kValues = mma_form(D, false, true);
            uint32_t keys_done = 0, pieces = 0, weights[2] = {};
            auto scores = [&](int stream, uint32_t key_tile) {
                const uint32_t q = q_at + stream * S::kOperand, k = k_at + key_tile % NB * S::kOperand;
                if (wait.lost) return;
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    const uint32_t off = (i >> 2) * 16384 + (i & 3) * 32;
                    tcgen05_mma_ss(tmem + stream * 128, smem_operand(q + off), smem_operand(k + off), kScores, i > 0);
                }
                mbar_arrive(smem_addr(&sh.s_full[stream]));
                tcgen05_commit(smem_addr(&sh.s_full[stream]));
            };
            auto values = [&](int stream, uint32_t key_tile, bool first) {
                const uint32_t v = v_at + key_tile % NB * S::kOperand;
                wait.one(sh.p_full[stream], weights[stream]++ & 1);
                tcgen05_after_sync();
                if (wait.lost) return;
#pragma unroll
                for (int i = 0; i < kChunkTile / 16; ++i)
                    tcgen05_mma_ts(tmem + 256 + stream * D, tmem + stream * 128 + 8 * i, smem_operand(v + i * 2048, 16384), kValues, !first || i > 0);
            };
            auto commit = [&](const unsigned long long& bar) {
                if (!wait.lost) tcgen05_commit(smem_addr(&bar));
            };
            auto key_ready = [&](uint32_t key_tile) {
                wait.one(sh.k_full[key_tile % NB], key_tile / NB & 1);
                tcgen05_after_sync();
            };
            while (walk.next(a, sh.lens, per_tile, p)) {
                const int n = p.end - p.begin;
                if (n == 0) continue;
                wait.one(sh.q_full[0], pieces & 1);
                wait.one(sh.q_full[1], pieces & 1);
                ++pieces;
                tcgen05_after_sync();
                const uint32_t g = keys_done;
                key_ready(g);
                scores(0, g);
                if constexpr (!SPLIT) scores(1, g);
                commit(sh.k_empty[g % NB]);
                if constexpr (SPLIT)
                    if (n > 1) {
                        key_ready(g + 1);
                        scores(1, g + 1);
                        commit(sh.k_empty[(g + 1) % NB]);
                    }
                for (int j = 0; j < n; ++j) {
                    const uint32_t now = g + j;
                    wait.one(sh.v_full[now % NB], now / NB & 1);
                    tcgen05_after_sync();
                    if constexpr (!SPLIT) {
                        values(0, now, j == 0);
                        if (j + 1 < n) {
                            key_ready(now + 1);
                            scores(0, now + 1);
                        } else commit(sh.o_full[0]);
                        values(1, now, j == 0);
                        commit(sh.v_empty[now % NB]);
                        if (j + 1 < n) {
                            scores(1, now + 1);
                            commit(sh.k_empty[(now + 1) % NB]);
                        } else commit(sh.o_full[1]);
                    } else {
                        const int stream = j & 1;
                        values(stream, now, j < 2);
                        commit(sh.v_empty[now % NB]);
                        if (j + 2 < n) {
                            key_ready(now + 2);
                            scores(stream, now + 2);
                            commit(sh.k_empty[(now + 2) % NB]);
                        } else commit(sh.o_full[stream]);
                    }
                }
                if (SPLIT && n == 1) commit(sh.o_full[1]);
                keys_done += n;
            }
            commit(sh.done);
            wait.one(sh.done, 0);
        }
        __syncwarp();
    } else {
        // ---- loader
        fence_proxy_async_global();                                    // (the records were written by ordinary stores)
        uint32_t keys_done = 0;
        while (walk.next(a, sh.lens, per_tile, p)) {
            const int b = a.s.b[p.u.seq];
            for (int j0 = p.begin; j0 < p.end; j0 += 16) {             // the pages of 16 tiles, one a lane
                const int j = j0 + lane / 2, page = p.u.tile(min(j, p.end - 1)) * 2 + lane % 2;
                int at = -1;                                           // (none)
                if (j < p.end && page < a.c.max_pages && page * kPageTokens < p.u.hi) at = a.c.page_table[(size_t)b * a.c.max_pages + page];
                if (at >= a.c.n_pages) at = -1;
                for (int i = 0; i < 16 && j0 + i < p.end; ++i, ++keys_done) {
                    const int at0 = __shfl_sync(0xffffffffu, at, 2 * i), at1 = __shfl_sync(0xffffffffu, at, 2 * i + 1);
                    const int stage = keys_done % S::kStages;
                    wait(sh.raw_empty[stage], keys_done / S::kStages & 1 ^ 1);
                    if (lane == 0 && !wait.lost) {
                        const uint32_t bar = smem_addr(&sh.raw_full[stage]), to = smem_addr(raw + stage * S::kRaw);
                        sh.raw_info[stage] = (at0 >= 0 ? 1u : 0u) | (at1 >= 0 ? 2u : 0u);
                        mbar_arrive_expect_tx(bar, ((at0 >= 0) + (at1 >= 0)) * 2u * S::kHalf);
                        if (at0 >= 0) bulk_g2s(to, a.c.pages + ((size_t)at0 * a.c.Hkv + p.head) * (2 * S::kHalf), 2 * S::kHalf, bar);
                        if (at1 >= 0) bulk_g2s(to + 2 * S::kHalf, a.c.pages + ((size_t)at1 * a.c.Hkv + p.head) * (2 * S::kHalf), 2 * S::kHalf, bar);
                    }
                    __syncwarp();
                }
            }
        }
        // copies in flight land before the block ends, also where the operands' warps have given up
        const uint32_t last = keys_done < (uint32_t)S::kStages ? keys_done : (uint32_t)S::kStages;
        for (uint32_t i = 0; i < last; ++i) {
            const uint32_t k = keys_done - 1 - i;
            wait(sh.raw_full[k % S::kStages], k / S::kStages & 1);
        }
    }
    tcgen05_before_sync();
    __syncthreads();
    tcgen05_after_sync();
    if (warp == 12) tmem_free(tmem);
}

// Units that the deal has cut: block x takes the one that starts in block x of the kernel above.
template <int D, bool SPLIT>
__global__ void __launch_bounds__(256) chunk_merge_kernel(const __grid_constant__ ChunkArgs a) {
    constexpr int kPerTile = chunk_rows(SPLIT), kQuads = D / 4;
    pdl_wait();
    pdl_launch_dependents();
    const ChunkCut cut = reinterpret_cast<const ChunkCut*>(a.workspace)[blockIdx.x];
    if (!cut.there) return;
    __shared__ int lens[kChunkBatch];
    if (threadIdx.x < a.s.n) lens[threadIdx.x] = max(a.c.seq_lens[a.s.b[threadIdx.x]], 0);
    __syncthreads();
    const int per_tile = SPLIT ? kPerTile / a.copies : kPerTile;
    const ChunkUnit u = chunk_unit(a, lens, cut.tile, per_tile);
    const float* slots = reinterpret_cast<const float*>(a.workspace + kChunkPlanBytes);
    constexpr size_t kSlot = chunk_slot_floats(D, SPLIT);
    auto part = [&](int k) { return slots + (size_t)(k == (int)blockIdx.x ? 2 * k + 1 : 2 * k) * kSlot; };
    for (int i = blockIdx.y * 256 + threadIdx.x; i < u.rows * kQuads; i += gridDim.y * 256) {
        const int row = i / kQuads, c = i % kQuads * 4;
        float most = -1e30f;
        for (int k = blockIdx.x; k <= cut.last; ++k) most = fmaxf(most, part(k)[kPerTile * D + row]);
        float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        float l = 0.0f;
#pragma unroll 4
        for (int k = blockIdx.x; k <= cut.last; ++k) {
            const float* s = part(k);
            const float r = ex2_approx(s[kPerTile * D + row] - most);
            const float4 x = *reinterpret_cast<const float4*>(s + (size_t)row * D + c);
            l += s[kPerTile * (D + 1) + row] * r;
            o.x += x.x * r, o.y += x.y * r, o.z += x.z * r, o.w += x.w * r;
        }
        const float inv = l > 0.0f ? __fdiv_rn(1.0f, l) : l == 0.0f ? 0.0f : l;
        uint16_t* out = static_cast<uint16_t*>(a.O) + chunk_row(a, u, cut.head, row) * D + c;
        *reinterpret_cast<uint2*>(out) = make_uint2(chunk_out(o.x * inv, o.y * inv, a.bf16), chunk_out(o.z * inv, o.w * inv, a.bf16));
    }
}

template <int D, int FMT, bool SPLIT>
cudaError_t launch_chunk(const ChunkArgs& a, int blocks, cudaStream_t s) {
    static OncePerDevice once;
    if (!allow_shared(chunk_kernel<D, FMT, SPLIT>, ChunkShape<D, FMT>::kBytes, once)) return cudaGetLastError();
    const cudaError_t e = launch_pdl(chunk_kernel<D, FMT, SPLIT>, dim3(blocks), dim3(kChunkThreads), (size_t)ChunkShape<D, FMT>::kBytes, s, a);
    if (e != cudaSuccess) return e;
    return launch_pdl(chunk_merge_kernel<D, SPLIT>, dim3(blocks, SPLIT ? 4 : 16), dim3(256), 0, s, a);
}

cudaError_t launch_chunk_pot(int d, int fmt, bool split, const ChunkArgs& a, int blocks, cudaStream_t s);
cudaError_t launch_chunk_plain(int d, int fmt, bool split, const ChunkArgs& a, int blocks, cudaStream_t s);

}  // namespace sa
