// Attention of several new tokens per sequence over the paged cache (sa_chunk_attention): the kernel.
//
// O = softmax(Q K^T / sqrt(d)) V for the last n tokens of a sequence, over every kind of cache, each token over what is not behind it, or over a
// window and the first few tokens.  The rows of a product are (token, query head of the KV head's group) pairs, so that a group's heads share a tile of keys.
//
// A block (one per SM) walks through pieces: 128 or 256 rows of one (sequence, KV head) and a stretch of tiles of 128 keys.  Its warps:
//   softmax    two streams of products, of 4 warps each (8 at head_dim 64): a row a thread, or half a row's columns;
//   operands   turn the records of a tile into operands, 16 bits a number: a key's code (PoT: bfloat16, INT8, 4 bits, binary16: binary16) without its
//              scale, which the softmax applies in FP32 to the scores, and values as the binary16 numbers that the codes stand for: both exact, as the
//              decode kernels' operands are;
//   products   one warp issues them (tcgen05): S = Q K^T into tensor memory, O += P V with the weights P read from there;
//   loader     copies the pages' records as they are into a ring in shared memory (bulk copies);
//   the deal   works out the block's pieces and hands them to the others through a ring, several ahead.
// The two streams take turns, so that the tensor core works on one while the softmax works on the other: two tiles of 128 rows
// against the same keys; or, where a sequence has no more than 128 rows (SPLIT), the same rows against every other tile of keys.  Of few rows a tile of
// 128 is filled up with copies, each for a part of the tile's keys (a thread then has 32 or 64 scores of a tile, not 128); the parts' sums meet at the end.
//
// Statistics and sums are FP32.  A weight is 2^(z - M + 7), z the logit in the log2 domain and M a reference that follows the row's maximum once that has grown by
// 8 (the sums are rescaled then): weights stay below 2^15, and what is 2^-21 of the largest keeps its 11 bits as a binary16 number.  That rounding, 2^-12 on
// average and independent from key to key, costs an output no more than its own rounding to binary16 does.
//
// Work is dealt on the device, as only that knows the lengths: units (KV head, sequence, row tile) in order, each with its tiles and a fixed cost, are cut into
// equal stretches, one a block.  A unit that a cut goes through leaves partial sums in the workspace, two places a block, for chunk_merge_kernel.  Where there are no more units
// than blocks and the longest is not much more than an equal stretch, a block has a unit and none is cut.
//
// What bounds it (in a CUDA graph; TFLOP/s of products that are needed):
//   head_dim 64, many rows: the powers.  256 rows x 128 keys take 2048 cycles of the unit for 2^x and about 3600 in all: it is busy for 63 %, issue slots for 62 %, the tensor core for 30 %.
//     2048 tokens over 32 768 PoT-M4 keys, 32 / 4 heads: 806 us, 660 TFLOP/s (585 with the powers left out, 528 with the codes' conversion left out as well).
//   head_dim 128, many rows: products (2050 cycles a tile at the rate of a library's) and powers (2048) beside one another.  8192 tokens, 32 / 8 heads, 4 bits: 517 us,
//     1060 TFLOP/s, 65 % of that rate; 4096 tokens over binary16 keys 168 us.
//   few rows (SPLIT): the way of a tile through the warps, each of which waits for the one before: 1400 cycles a tile, where 730 are what memory needs, and all but 200 of them
//     stay when powers and conversion are left out.  32 single tokens over 32 768 PoT-M4 keys: 169 us, 3.3 TB/s.
//   one short call: what it takes to get going, 7 us: lengths, deal, page table, records, operands, one product after another, outputs.
#pragma once
#include <cuda_bf16.h>
#include <type_traits>

#include "sa_cache_write.cuh"
#include "sa_common.cuh"
#include "sa_fp4.cuh"
#include "sa_score_mma.cuh"
#include "sa_stage.cuh"
#include "sa_tcgen05.cuh"

namespace sa {

constexpr int kChunkBatch = 128;          // sequences per launch
constexpr int kChunkTile = 128;           // keys
constexpr int kChunkUnitCost = 4;         // what a unit costs beside its tiles, in tiles
// What cutting units costs, in tiles, beside a kernel of a unit a block: a second start in most blocks, partial sums, putting them together.  (As many tiles as the longest unit has more than
// an equal stretch where both take equally long, 4 to 136 equal units and causal ones: few rows at head_dim 64 8 to 10 tiles, 8 sequences of 1024 tokens 15.9 us cut, 15.6 whole, of 2048 17.6
// and 21.3; the others 7 to 8, 1024 new tokens of 16 / 2 heads of 128 34.6 and 36.9, 512 27.9 and 26.4.)
SA_HD constexpr int chunk_cut_cost(int d, bool split) { return split && d == 64 ? 9 : 7; }
constexpr int kChunkBlocksMost = 1024;
constexpr int kChunkCutBytes = kChunkBlocksMost * 96;      // of the workspace, ahead of the partial sums: the piece of every block that the cut behind it goes through
SA_HD constexpr int chunk_rows(bool split) { return split ? 128 : 256; }
SA_HD constexpr size_t chunk_slot_floats(int d, bool split) { return (size_t)chunk_rows(split) * (d + 2); }

struct ChunkSeqs {
    int n;                                // sequences of this launch
    int b[kChunkBatch];                   // each: its number in the cache
    int tokens[kChunkBatch];              // new tokens, and their first row in Q and O
    int64_t row0[kChunkBatch];
    int tiles[kChunkBatch + 1];           // row tiles ahead of it
};
// x / d for 0 <= x < 2^31 by a product (Granlund and Montgomery): with 2^s >= d, mul = floor(2^(31 + s) / d) + 1 is above the quotient by at most 1, the product by less than 1 / d.
struct ChunkDivisor {
    uint32_t mul;
    int shift;
    ChunkDivisor() = default;
    explicit ChunkDivisor(int d) : mul(0), shift(31) {
        while ((1ll << (shift - 31)) < d) ++shift;
        mul = (uint32_t)((1ull << shift) / (uint64_t)d + 1);
    }
    SA_HD int operator()(int x) const { return (int)((uint64_t)(uint32_t)x * mul >> shift); }
};
struct ChunkArgs {
    CacheArgs c;
    ChunkDivisor by_group;                // rows (token, query head of the group) to tokens
    const uint16_t* Q;
    void* O;
    uint8_t* workspace;
    int Hq, G, window, sinks;             // G: query heads of a group
    int copies;                           // SPLIT: 1, 2 or 4 copies of the rows in a tile
    int whole, merged;                    // a unit a block, whatever the lengths: none is cut; else the deal decides: chunk_merge_kernel follows
    int bf16;                             // type of O
    int lost_b, lost_head, lost_tile;     // LOST (sa_debug_chunk_lost_copy)
    float factor;                         // log2(e) / sqrt(d) and the unit of the operands
    ChunkSeqs s;
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
    u.first = before + a.by_group(u.row0);
    u.last = before + a.by_group(u.row0 + u.rows - 1);
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

// A piece of a block's work as its warps read it, in shared memory.
struct ChunkPiece {
    int n;                                // key tiles; -1: no more pieces
    int head, b;
    int rows, token_row, token;           // row r is row token_row + r of the heads of the group, counted from token `token` (of the sequence) on
    int64_t q_token;                      // that token's row in Q and O
    int lo, hi;                           // keys lo .. hi - 1, and below sinks
    int sink_tiles, window_tile, begin;   // of the unit; the piece's first tile
    int place;                            // 0: the whole unit; 1, 2: its sums go to the block's first, second place,
    int last_block;                       // 2: the unit's other parts are in the first places of the blocks up to this one
    int first[2], last[2];                // of the streams: positions of the first and last row's token
    SA_D int tile(int i) const { return begin + i < sink_tiles ? begin + i : window_tile + begin + i - sink_tiles; }
    // Row r: its token's position, its row (of heads) in Q and O.
    SA_D int position(const ChunkArgs& a, int r) const { return token + a.by_group(token_row + r); }
    SA_D int64_t row(const ChunkArgs& a, int r) const {
        const int at = token_row + r, t = a.by_group(at);
        return (q_token + t) * a.Hq + head * a.G + (at - t * a.G);
    }
};
static_assert(sizeof(ChunkPiece) <= 96, "room in the workspace");
SA_D ChunkPiece* chunk_cut(const ChunkArgs& a, int block) { return reinterpret_cast<ChunkPiece*>(a.workspace + block * 96); }
// The sums that a piece leaves at place 1 or 2 of its block: [rows][D] outputs, references, sums of weights.
template <int D, bool SPLIT>
SA_D float* chunk_slot(const ChunkArgs& a, int block, int place) {
    return reinterpret_cast<float*>(a.workspace + kChunkCutBytes) + (size_t)(2 * block + place - 1) * chunk_slot_floats(D, SPLIT);
}
constexpr int kChunkPieces = 8;           // of them in the ring, as the loader may be several ahead

// Warps of a block, and registers of their threads: what the block is launched with and what the groups of four warps then have of it.
//   softmax   two streams of 4 warps, a row a thread; at head_dim 64 of 8, half a row's columns a thread: there the powers bound the kernel, and twice the warps hide more of what
//             is around them (2048 tokens over 32 768 PoT-M4 keys 834 -> 777 us); at 128 the two threads' meeting costs more than that (a prompt of 8192 tokens, 4 bits, 549 -> 583);
//   operands  4 warps, a key a thread (SPLIT, where little else is done with a tile: 4 for keys and 4 for values, of every other tile, twice: 209 -> 184 us of 32 single
//             tokens over 32 768 keys);
//   others    products, loader, the one that deals, an idle one.
template <int D, bool SPLIT>
struct ChunkForm {
    static constexpr int kHalves = SPLIT || D == 128 ? 1 : 2;         // threads of a row
    static constexpr int kSoftmax = 8 * kHalves, kOperand = SPLIT ? 16 : 4, kThreads = 32 * (kSoftmax + kOperand + 4);
    static constexpr int kLaunch = SPLIT ? 72 : kHalves == 2 ? 80 : 128;
    static constexpr int kSoftmaxRegs = SPLIT ? 120 : kHalves == 2 ? 96 : 192, kOperandRegs = SPLIT || kHalves == 2 ? 56 : 72, kOtherRegs = SPLIT || kHalves == 2 ? 40 : 56;
    static_assert(32 * (kSoftmax * kSoftmaxRegs + kOperand * kOperandRegs + 4 * kOtherRegs) <= kThreads * kLaunch && kThreads * kLaunch <= 65536, "the groups' registers are those of the launch");
};

// Shared memory of a block.
template <int D, int FMT>
struct ChunkShape {
    static constexpr int kHalf = FMT == FMT_FP16 ? half_block_bytes_fp16(D) : FMT == FMT_FP4 ? half_block_bytes_fp4(D)
                                 : half_block_bytes(D, FMT == FMT_PLANAR1 ? 1 : FMT == FMT_PLANAR2 ? 2 : FMT == FMT_INT8 ? 8 : 0, FMT == FMT_NIBBLE || FMT == FMT_PLANAR1 || FMT == FMT_PLANAR2);
    static constexpr int kRaw = 4 * kHalf;                            // records of a tile
    static constexpr int kOperand = D / 64 * 16384;                   // 128 rows
    static constexpr int kBuffers = D == 64 ? 2 : 1;                  // of operands
    static constexpr int kFixed = (2 + 2 * kBuffers) * kOperand + 14336;
    static constexpr int kFit = (227 * 1024 - 1024 - kFixed) / kRaw;
    static constexpr int kStages = kFit >= 8 ? 8 : kFit >= 6 ? 6 : kFit > 4 ? 4 : kFit;      // (4 to 8: 32 single tokens over 32 768 keys 178 -> 172 us)
    static constexpr int kBytes = 1024 + kFixed + kStages * kRaw;     // (1024: to align)
    static constexpr int kRing = kStages % 2 ? 2 * kStages : kStages;  // barriers of the records: an even number, so that warps which take every other tile see all phases of theirs
    static constexpr int kV = (FMT == FMT_FP16) ? 64 * D : FMT == FMT_FP4 ? 18 * D : kHalf - 32 * D;      // offset of the values in a half
    static constexpr int kMeta = FMT == FMT_FP4 ? 16 * D : kV - 128;
    static constexpr bool kScaled = FMT != FMT_FP16 && FMT != FMT_FP4;                                  // keys have a scale of their own
    static constexpr bool kBf16 = kScaled && FMT != FMT_INT8;                                           // type of keys and queries
    static_assert(kStages >= 1, "a tile's records have to fit");
    // Columns of tensor memory: scores of the streams, 128 each; sums; at head_dim 64 the weights have a place of their own, so that the next tile's scores are
    // under way while the softmax works on the last one's; at 128 they take the scores'.
    static constexpr bool kApart = D == 64;
    SA_HD static constexpr uint32_t weights(int stream) { return kApart ? 384 + 64 * stream : 128 * stream; }
    SA_HD static constexpr uint32_t sums(int stream) { return 256 + D * stream; }
};
struct ChunkShared {                      // behind the rings
    // Of eight tiles.  Tile j's place is written once the products of the scores of tile j - 2 (head_dim 128: j - 1) are done, which are issued when the softmax has read the scores of the
    // tile before in their stream: it may be at tile j - 5 then, no further back (SPLIT; else at j - 3).
    float scale[8][kChunkTile];           // of the keys
    float m[256], l[256];                 // SPLIT: of all threads' rows
    float meet[3][512];                   // else: what the two halves of a row tell each other
    int2 info[8];                         // raw_info
    ChunkPiece pieces[kChunkPieces], undealt;
    unsigned long long piece_full[kChunkPieces], piece_empty[kChunkPieces];
    int2 raw_info[8];                     // of a place of records: first key; bits 0, 1: which of the tile's pages there are, 2, 3: streams whose rows see all of the tile, 4: some row sees each key
    unsigned long long raw_full[8], raw_empty[8], k_full[2], k_empty[2], v_full[2], v_empty[2], q_full[2], s_full[2], s_free[2], p_full[2], o_full[2], done;
    int lens[kChunkBatch];
    uint32_t tmem;
};
static_assert(sizeof(ChunkShared) <= 14336, "room behind the rings");

// A wait that ends: where the limit is reached (kWaitLimit polls, which sleep for up to 4 us each: a second; LONGER of them where a whole piece is waited for) the warp waits for nothing
// any more: what it makes from there on goes into no product, and the rows of its block's pieces, this one and those that follow, become NaN (the deal: those that it hands out no more).
// LOST: the kernel of sa_debug_chunk_lost_copy, where some waits do run out, with a limit of a few ms.  (With a shorter sleep asked for, each poll is a loop of several instructions: a prompt of 8192 tokens, 4 bits, 547 us, not 531.)
template <uint32_t LONGER, bool LOST>
struct ChunkWait {
    static constexpr uint32_t kPolls = LONGER * (LOST ? 1u << 10 : kWaitLimit);
    bool lost = false;
    SA_D static bool poll(uint32_t bar, uint32_t parity) {
        uint32_t ok;
        asm volatile("{.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
        return ok != 0;
    }
    SA_D static bool over(uint32_t bar, uint32_t parity) {                      // (the phase is over already: a look that cannot sleep is the faster one)
        uint32_t ok;
        asm volatile("{.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
        return ok != 0;
    }
    SA_D void operator()(const unsigned long long& bar, uint32_t parity) {      // by a whole warp
        const uint32_t at = smem_addr(&bar);
        if (!over(at, parity) && !lost) {
            lost = true;
#pragma unroll 1
            for (uint32_t i = 0; i < kPolls && lost; ++i) lost = !poll(at, parity);
        }
        __syncwarp();
    }
};

// The pieces, one after another: next() gives the one at hand (null: no more), leave() hands its place back.  By a whole warp.  (Its waits are its own: warps that have given
// up on a tile go on from piece to piece, and write the NaN.  They run out where the deal has given up, all warps' together; it waits for 16 limits, more than the other warps take to give up
// on whatever they wait for, so that takes a warp that makes no way at all.)
template <bool LOST>
struct ChunkReader {
    ChunkShared& sh;
    ChunkWait<32, LOST> wait{};
    uint32_t i = 0;
    SA_D const ChunkPiece* next() {
        wait(sh.piece_full[i % kChunkPieces], i / kChunkPieces & 1);
        const ChunkPiece* p = &sh.pieces[i % kChunkPieces];
        return __any_sync(0xffffffffu, wait.lost) || p->n < 0 ? nullptr : p;
    }
    SA_D void leave() {
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive(smem_addr(&sh.piece_empty[i % kChunkPieces]));
        ++i;
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

// INT8 values 2 I, 2 I + 1 of a word as binary16 numbers 1152 larger: the biased byte in the low mantissa bits of 1024.
template <int I>
SA_D uint32_t int8_biased(uint32_t w) { return __byte_perm(w ^ 0x80808080u, 0x64646464u, I ? 0x4342u : 0x4140u); }
SA_D uint32_t add_half2_1152(uint32_t h) {
    asm("add.rn.f16x2 %0, %0, %1;" : "+r"(h) : "r"(0xe480e480u));
    return h;
}
SA_D uint32_t fma_half2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
SA_D uint32_t twice_half(float x) { return (uint32_t)__half_as_ushort(__float2half_rn(x)) * 0x10001u; }
// The codes of one token's key (KEY) or value (t of a half): read at once, then put into a row of the operand (zeros: not seen).
template <int D, int FMT, bool KEY>
struct ChunkCodes {
    using S = ChunkShape<D, FMT>;
    static constexpr bool kPairs = FMT == FMT_FP4 && !KEY;             // 4-bit values: a byte is two tokens' nibbles
    static constexpr int kPlanes = !KEY ? 0 : FMT == FMT_PLANAR1 ? 1 : FMT == FMT_PLANAR2 ? 2 : 0;
    static constexpr bool kNibbles = KEY && (FMT == FMT_NIBBLE || FMT == FMT_PLANAR1 || FMT == FMT_PLANAR2);
    static constexpr int kChunks = FMT == FMT_FP16 ? D / 8 : FMT == FMT_FP4 || kNibbles ? D / 32 : D / 16;
    static constexpr int kAhead = FMT == FMT_FP16 ? 4 : kChunks;       // chunks that are read ahead of the wait for the operand's place
    uint4 w[kPairs ? 1 : kAhead];
    uint32_t plane[kPlanes ? kPlanes * D / 32 : 1];

    SA_D static const uint4* chunk(const uint8_t* half, int t) { return reinterpret_cast<const uint4*>(half + (KEY ? 0 : S::kV)) + t; }      // + 32 k: chunk k
    SA_D ChunkCodes(const uint8_t* half, int t) {
        if constexpr (!kPairs) {
#pragma unroll
            for (int k = 0; k < kAhead; ++k) w[k] = chunk(half, t)[32 * k];
        }
#pragma unroll
        for (int bit = 0; bit < kPlanes; ++bit)
#pragma unroll
            for (int k = 0; k < D / 32; ++k) plane[bit * (D / 32) + k] = *reinterpret_cast<const uint32_t*>(half + 16 * D + (bit * kTileTokens + t) * (D / 8) + 4 * k);
    }
    SA_D void put(const uint8_t* half, int t, uint32_t operand, int row, bool seen) {
        auto to = [&](int c, uint32_t a, uint32_t b, uint32_t x, uint32_t y) { put_operand(operand, row, c, a, b, x, y); };
        if constexpr (FMT == FMT_FP16) {
#pragma unroll
            for (int c = 0; c < D / 8; ++c) {
                const uint4 v = w[c % kAhead];
                if (c + kAhead < D / 8) w[c % kAhead] = chunk(half, t)[32 * (c + kAhead)];
                to(c, v.x, v.y, v.z, v.w);
            }
        } else if constexpr (kPairs) {
            const uint8_t* at = half + S::kV + t % 8 / 2 * 16 + t / 16 * 4 + t / 8 % 2 * 2;
            const uint8_t* scales = half + S::kV + 16 * D + t % 8 / 2 * 16 + t / 16 * 4 + t % 2 * 2 + t / 8 % 2;
            const int shift = 4 * (t & 1);
            uint32_t x[2][8], b[2];                                                     // of this block of 16 channels and the next: x[e]: channels e, e + 8
            auto read = [&](int blk) {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[blk % 2][e] = *reinterpret_cast<const uint16_t*>(at + blk / 2 * 512 + e * 64 + blk % 2 * 8);
                b[blk % 2] = scales[blk / 2 * 64 + blk % 2 * 8];
            };
            read(0);
#pragma unroll
            for (int blk = 0; blk < D / 16; ++blk) {
                if (blk + 1 < D / 16) read(blk + 1);
                uint32_t n[8], h[4];
#pragma unroll
                for (int e = 0; e < 8; ++e) n[e] = x[blk % 2][e] >> shift & 0x0f0fu;
#pragma unroll
                for (int e = 0; e < 8; e += 2) n[e] |= n[e + 1] << 4;
                const uint32_t lo = n[0] | n[2] << 16, hi = n[4] | n[6] << 16, s = b[blk % 2] << 7 | b[blk % 2] << 23;
                const uint32_t word[2] = {__byte_perm(lo, hi, 0x6420), __byte_perm(lo, hi, 0x7531)};
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    fp4_to_half2(word[i], h);
                    to(2 * blk + i, mul_half2(h[0], s), mul_half2(h[1], s), mul_half2(h[2], s), mul_half2(h[3], s));
                }
            }
        } else if constexpr (FMT == FMT_FP4) {
            uint32_t b[D / 16];
#pragma unroll
            for (int i = 0; i < D / 16; ++i) b[i] = half[16 * D + i / 4 * 128 + i % 4 * 32 + t % 8 * 4 + t / 8];
#pragma unroll
            for (int k = 0; k < D / 32; ++k) {
                const uint32_t code[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t s = b[k / 2 * 4 + i] << 7 | b[k / 2 * 4 + i] << 23;
                    uint32_t h[4];
                    fp4_to_half2(code[i], h);
                    to(8 * (k / 2) + 2 * i + k % 2, mul_half2(h[0], s), mul_half2(h[1], s), mul_half2(h[2], s), mul_half2(h[3], s));
                }
            }
        } else if constexpr (KEY && !kNibbles) {
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                const uint32_t code[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
                uint32_t h[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (FMT == FMT_BYTE) {
                        h[2 * i] = byte_codes_to_bf16<0>(code[i], 1u);
                        h[2 * i + 1] = byte_codes_to_bf16<2>(code[i], 1u);
                    } else {
                        h[2 * i] = add_half2_1152(int8_biased<0>(code[i]));
                        h[2 * i + 1] = add_half2_1152(int8_biased<1>(code[i]));
                    }
                }
                to(2 * k, h[0], h[1], h[2], h[3]);
                to(2 * k + 1, h[4], h[5], h[6], h[7]);
            }
        } else if constexpr (KEY) {
#pragma unroll
            for (int k = 0; k < D / 32; ++k) {
                const uint32_t code[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t h[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        h[i] = nibbles_to_bf16(code[c], i);
                        if constexpr (kPlanes == 1) h[i] |= plane_pair<6>(plane[k] >> (8 * c), i);
                        if constexpr (kPlanes == 2) h[i] |= plane_pair<5>(plane[k] >> (8 * c), i) | plane_pair<6>(plane[D / 32 + k] >> (8 * c), i);
                    }
                    to(4 * k + c, h[0], h[1], h[2], h[3]);
                }
            }
        } else {
            // times 2^-g in two exact steps: the first (with the bias of the bytes taken off) keeps clear of the subnormal and of the largest numbers; the product is a number that
            // binary16 has, as the value that was rounded was one, but for 65536, which becomes the largest
            const int g = (int)(int8_t)half[S::kMeta + t * 4 + 2], g1 = max(-5, min(g, 12));
            const uint32_t f1 = twice_half(pow2i(-g1)), off = twice_half(-1152.0f * pow2i(-g1)), f2 = twice_half(pow2i(max(g1 - g, -40)));
            const bool twice = __any_sync(0xffffffffu, g != g1);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                const uint32_t code[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
                uint32_t h[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    h[2 * i] = fma_half2(int8_biased<0>(code[i]), f1, off);
                    h[2 * i + 1] = fma_half2(int8_biased<1>(code[i]), f1, off);
                }
                if (twice) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        h[i] = mul_half2(h[i], f2);
                        asm("{.reg .b32 m; mov.b32 m, 0x7bff7bff; min.f16x2 %0, %0, m; neg.f16x2 m, m; max.f16x2 %0, %0, m;}" : "+r"(h[i]));
                    }
                }
                to(2 * k, h[0], h[1], h[2], h[3]);
                to(2 * k + 1, h[4], h[5], h[6], h[7]);
            }
        }
        if (!seen) {
#pragma unroll 1
            for (int c = 0; c < D / 8; ++c) to(c, 0u, 0u, 0u, 0u);
        }
    }
};

// 32 queries (HALVES = 2: the first or, with half = 1, the last 16 of them) as rows of the operand, D / 16 lanes a row; returns the factor of the lane's own row, if it is one of
// them.  row_of(r): row r's binary16 numbers, or null.
template <int D, int FMT, int HALVES, typename RowOf>
SA_D float chunk_queries(const ChunkArgs& a, uint32_t operand, int lane, int first_row, int half, RowOf row_of) {       // (rows behind the last one are zeros: whole steps of them cost little)
    using S = ChunkShape<D, FMT>;
    constexpr int LPV = D / 16, RPW = 32 / LPV, STEPS = 32 / RPW / HALVES;
    const int row0 = half * STEPS * RPW;
    const Fp4Half<D> f(lane, 0);
    uint32_t x[STEPS][8];
    bool any[STEPS];
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const uint16_t* p = row_of(row0 + i * RPW + lane / LPV);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] = 0u;
        if (p) load_32_bytes(p + 16 * f.blk, (reinterpret_cast<uintptr_t>(a.Q) & 31) == 0, x[i]);
        any[i] = __any_sync(0xffffffffu, p != nullptr);
    }
    float mine = a.factor;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        if (a.c.hadamard && any[i]) f.rotate(x[i]);
        // A query with an infinity or a NaN is a NaN in the operand, and scores are NaN where a key is seen and nowhere else: in the factor it would be in hidden keys' weights too, and
        // an infinity can make all scores minus infinity, which reads as nothing seen.
        if (S::kScaled && any[i]) {                                                     // as quantise_query_vec: 127 steps of the largest magnitude
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
            const bool number = top < 0x7c00u;
            if (!number) x[i][0] = 0x7fff7fffu;
            const float d = __shfl_sync(0xffffffffu, top && number ? delta : 1.0f, (lane % RPW) * LPV);      // (a query of zeros: any factor but zero)
            if (lane / RPW == half * STEPS + i) mine = d * a.factor;
        } else if (any[i]) {
            uint32_t zero[2] = {mul_half2(x[i][0], 0u), mul_half2(x[i][1], 0u)};        // (or NaN)
#pragma unroll
            for (int e = 2; e < 8; ++e) zero[e & 1] = fma_half2(x[i][e], 0u, zero[e & 1]);
            x[i][0] = fma_half2(zero[0], 0u, fma_half2(zero[1], 0u, x[i][0]));
        }
        const int row = first_row + row0 + i * RPW + lane / LPV;
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
// Outputs are means of numbers that binary16 has, but the weights are rounded and the sum that they are divided by is not: a mean of values of the largest magnitude, 65504, may come out
// as up to 2^-11 more, which rounds to infinity.  So sums whose output would be 65520 or more, and are no infinities, are cut down to 65504 times the row's sum of weights.
constexpr float kChunkRoundsUp = 65520.0f;
SA_D float chunk_cut_down(float x, float l) { return fabsf(x) < INFINITY ? fminf(fmaxf(x, -65504.0f * l), 65504.0f * l) : x; }
SA_D float max3_abs(float a, float b, float c) {
    float d;
    asm("max.abs.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// Four outputs: sums of a row whose weights' sum is l.
SA_D uint2 chunk_out4(float4 v, float l, int bf16) {
    const float inv = l > 0.0f ? __fdiv_rn(1.0f, l) : l == 0.0f ? 0.0f : l;
    if (!bf16 && max3_abs(max3_abs(v.x, v.y, v.z), v.w, 0.0f) * inv >= kChunkRoundsUp)
        v = make_float4(chunk_cut_down(v.x, l), chunk_cut_down(v.y, l), chunk_cut_down(v.z, l), chunk_cut_down(v.w, l));
    return make_uint2(chunk_out(v.x * inv, v.y * inv, bf16), chunk_out(v.z * inv, v.w * inv, bf16));
}
SA_D uint32_t bits_below(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }
SA_D void chunk_sync(int barrier, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(threads) : "memory"); }

template <int N>
SA_D void registers_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
SA_D void registers_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// A row's softmax: reference and sum of weights (in its units), factor from a product's units to the log2 domain.
struct ChunkRow {
    float m, l, factor;
};
// Which columns of a tile (whose first key is t0) a row sees.
struct ChunkMask {
    int t0, pages, position, window, sinks;
};
SA_D float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// 32 columns of a row's scores, in registers x: times the keys' scales.
template <int D, int FMT>
SA_D void chunk_scores(const uint32_t (&x)[32], f32x2 (&y)[16], const float* scale, int c) {
#pragma unroll
    for (int e = 0; e < 16; ++e) y[e] = pack_f32x2(__uint_as_float(x[2 * e]), __uint_as_float(x[2 * e + 1]));
    if constexpr (ChunkShape<D, FMT>::kScaled) {
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            const float4 s4 = *reinterpret_cast<const float4*>(scale + 32 * c + 2 * e);
            y[e] = mul2(y[e], pack_f32x2(s4.x, s4.y));
            y[e + 1] = mul2(y[e + 1], pack_f32x2(s4.z, s4.w));
        }
    }
}
// Scores of hidden keys become -inf where they lie, in tensor memory: few tiles need it, and in registers the others would pay for the meeting of the branches
// with a move of every score.
SA_D void chunk_hide(const ChunkMask& mask, uint32_t s_col, int chunk0, int chunks) {
    const int hi = mask.position - mask.t0, sink = mask.sinks - mask.t0;
    const int lo = mask.window && mask.position >= 0 ? (int)max((long long)hi - mask.window + 1, -0x40000000ll) : -0x40000000;
#pragma unroll 1
    for (int c = chunk0; c < chunk0 + chunks; ++c) {
        uint32_t x[32];
        tmem_load(s_col + 32 * c, x);
        tmem_loaded();
        const int at = 32 * c;
        const uint32_t seen = (mask.pages >> (c >> 1) & 1u) ? bits_below(hi - at + 1) & (~bits_below(lo - at) | bits_below(sink - at)) : 0u;
#pragma unroll
        for (int e = 0; e < 32; ++e) x[e] = seen >> e & 1u ? x[e] : 0xff800000u;
        tmem_store(s_col + 32 * c, x);
    }
    tmem_stored();
}
SA_D void chunk_largest(const f32x2 (&y)[16], float (&top)[4]) {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        float v, w;
        unpack_f32x2(y[e], &v, &w);
        top[e & 3] = max3(top[e & 3], v, w);
    }
}
// The reference follows the largest score; returns what the sums so far are worth in its units.
SA_D float chunk_reference(ChunkRow& row, float top, bool& grown) {
    const float z = top * row.factor;
    grown = z > row.m + 8.0f;
    const float shrink = grown ? ex2_approx(row.m - z) : 1.0f;
    if (grown) row.m = z;
    row.l *= shrink;
    return shrink;
}
// Weights of 32 columns, and their sum to l (of the numbers ahead of their rounding: with the sum of the rounded ones outputs are no nearer, and a fifth more instructions).
SA_D void chunk_weights(const ChunkRow& row, f32x2 (&y)[16], uint32_t (&w)[16], f32x2 (&l)[2]) {
    const f32x2 f2 = pack_f32x2(row.factor, row.factor), m2 = pack_f32x2(7.0f - row.m, 7.0f - row.m);
#pragma unroll
    for (int e = 0; e < 16; ++e) y[e] = ffma2(y[e], f2, m2);
#pragma unroll
    for (int b = 0; b < 16; b += 4) {
#pragma unroll
        for (int e = b; e < b + 4; ++e) {
            float u0, u1;
            unpack_f32x2(y[e], &u0, &u1);
            y[e] = pack_f32x2(ex2_approx(u0), ex2_approx(u1));
        }
#pragma unroll
        for (int e = b; e < b + 4; ++e) {
            float u0, u1;
            unpack_f32x2(y[e], &u0, &u1);
            w[e] = half2_of(u0, u1);
            l[e & 1] = add2(l[e & 1], y[e]);
        }
    }
}
template <int D>
SA_D void chunk_shrink(uint32_t o_col, float shrink) {
#pragma unroll 1
    for (int c = 0; c < D; c += 16) {
        uint32_t o[16];
        tmem_load(o_col + c, o);
        tmem_loaded();
#pragma unroll
        for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * shrink);
        tmem_store(o_col + c, o);
    }
}
SA_D void chunk_scores_read(bool apart, uint32_t free_scores) {
    if (!apart) return;
    tcgen05_before_sync();
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(free_scores);
}
// One tile of a row: columns 32 chunk0 .. of the scores (32 C of them) to weights.  free_scores: mbarrier, where the scores' place is apart from the weights';
// ahead(): waits until weights and sums may be written; all(x): the largest x of the row's threads; sums: there are some, OUT channels of them from o_col for this thread to
// rescale.  TWICE: the scores are read once for the largest and again for the weights, by a thread without the registers for all of them.
template <int D, int FMT, int C, bool TWICE, int OUT, typename Ahead, typename All>
SA_D void chunk_softmax(ChunkRow& row, const float* scale, uint32_t s_col, uint32_t p_col, int chunk0, uint32_t free_scores, Ahead ahead, All all, bool sums, uint32_t o_col) {
    using S = ChunkShape<D, FMT>;
    float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    f32x2 l[2] = {pack_f32x2(0.0f, 0.0f), pack_f32x2(0.0f, 0.0f)};
    bool grown;
    if constexpr (TWICE) {
        uint32_t x[32], w[16];
        f32x2 y[16];
#pragma unroll 1
        for (int c = chunk0; c < chunk0 + C; ++c) {
            tmem_load(s_col + 32 * c, x);
            tmem_loaded();
            chunk_scores<D, FMT>(x, y, scale, c);
            chunk_largest(y, top);
        }
        const float shrink = chunk_reference(row, all(fmaxf(max3(top[0], top[1], top[2]), top[3])), grown);
        ahead();
        if (sums && __any_sync(0xffffffffu, grown)) chunk_shrink<OUT>(o_col, shrink);
#pragma unroll 1
        for (int c = chunk0; c < chunk0 + C; ++c) {                    // (weights in the scores' place: 16 c .. is behind what has been read)
            tmem_load(s_col + 32 * c, x);
            tmem_loaded();
            chunk_scores<D, FMT>(x, y, scale, c);
            chunk_weights(row, y, w, l);
            tmem_store(p_col + 16 * c, w);
        }
        chunk_scores_read(S::kApart, free_scores);
    } else {
        uint32_t x[C][32], w[C][16];
        f32x2 y[C][16];
#pragma unroll
        for (int c = 0; c < C; ++c) tmem_load(s_col + 32 * (chunk0 + c), x[c]);
        tmem_loaded();
        chunk_scores_read(S::kApart, free_scores);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            chunk_scores<D, FMT>(x[c], y[c], scale, chunk0 + c);
            chunk_largest(y[c], top);
        }
        const float shrink = chunk_reference(row, all(fmaxf(max3(top[0], top[1], top[2]), top[3])), grown);
#pragma unroll
        for (int c = 0; c < C; ++c) chunk_weights(row, y[c], w[c], l);
        ahead();
        if (sums && __any_sync(0xffffffffu, grown)) chunk_shrink<OUT>(o_col, shrink);
#pragma unroll
        for (int c = 0; c < C; ++c) tmem_store(p_col + 16 * (chunk0 + c), w[c]);
    }
    float l0, l1;
    unpack_f32x2(add2(l[0], l[1]), &l0, &l1);
    row.l += l0 + l1;
}

// The rows of a piece that is not handed out: NaN, or its place's sums of weights, so that no merge takes what an earlier call has left there.  By a whole warp.
template <int D, bool SPLIT>
SA_D void chunk_undealt(const ChunkArgs& a, const ChunkPiece& p, int lane) {
    const float nan = __int_as_float(0x7fc00000);
    if (p.place) {
        float* slot = chunk_slot<D, SPLIT>(a, blockIdx.x, p.place);
        for (int r = lane; r < p.rows; r += 32) {
            slot[chunk_rows(SPLIT) * D + r] = 0.0f;
            slot[chunk_rows(SPLIT) * (D + 1) + r] = nan;
        }
    } else {
        for (int i = lane; i < p.rows * (D / 8); i += 32)
            *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.O) + p.row(a, i / (D / 8)) * D + i % (D / 8) * 8) = make_uint4(0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu);
    }
    __threadfence();
}

template <int D, int FMT, bool SPLIT, bool LOST>
__global__ void __launch_bounds__(ChunkForm<D, SPLIT>::kThreads, 1) chunk_kernel(const __grid_constant__ ChunkArgs a) {
    using S = ChunkShape<D, FMT>;
    using Form = ChunkForm<D, SPLIT>;
    constexpr int kPerTile = chunk_rows(SPLIT), NB = S::kBuffers, kHalves = Form::kHalves, kOperands = Form::kSoftmax, kProducts = kOperands + Form::kOperand;      // (first warps)
    extern __shared__ uint8_t dynamic[];
    const uint32_t base = (smem_addr(dynamic) + 1023u) & ~1023u;
    uint8_t* const rings = dynamic + (base - smem_addr(dynamic));
    const uint32_t q_at = base, k_at = q_at + 2 * S::kOperand, v_at = k_at + NB * S::kOperand;
    uint8_t* const raw = rings + (2 + 2 * NB) * S::kOperand;
    ChunkShared& sh = *reinterpret_cast<ChunkShared*>(raw + S::kStages * S::kRaw);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int per_tile = SPLIT ? kPerTile / a.copies : kPerTile;

    if (tid == 0) {
        for (int i = 0; i < S::kRing; ++i) {
            mbar_init(smem_addr(&sh.raw_full[i]), 1);
            mbar_init(smem_addr(&sh.raw_empty[i]), SPLIT ? 8 : 4);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_addr(&sh.k_full[i]), 4);
            mbar_init(smem_addr(&sh.v_full[i]), 4);
            mbar_init(smem_addr(&sh.k_empty[i]), 1);
            mbar_init(smem_addr(&sh.v_empty[i]), 1);
            mbar_init(smem_addr(&sh.q_full[i]), 4 * kHalves);
            mbar_init(smem_addr(&sh.s_full[i]), 2);                    // (the products' arrival, and the issuing thread's own, which hands on what it has seen)
            mbar_init(smem_addr(&sh.s_free[i]), 4 * kHalves);
            mbar_init(smem_addr(&sh.p_full[i]), 4 * kHalves);
            mbar_init(smem_addr(&sh.o_full[i]), 1);
        }
        for (int i = 0; i < kChunkPieces; ++i) {
            mbar_init(smem_addr(&sh.piece_full[i]), 1);
            mbar_init(smem_addr(&sh.piece_empty[i]), Form::kSoftmax + Form::kOperand + 2);
        }
        mbar_init(smem_addr(&sh.done), 1);
        fence_mbar_init();
    }
    if (warp == kProducts) tmem_alloc(smem_addr(&sh.tmem));
    tcgen05_before_sync();
    __syncthreads();
    tcgen05_after_sync();
    pdl_wait();
    if (a.merged) pdl_launch_dependents();                             // (else a call behind this one that reads its output early would be too early)
    ChunkWait<1, LOST> wait;
    ChunkReader<LOST> reader{sh};

    if (warp < kOperands) {
        // ---- softmax: a row a thread, or half a row's columns
        const int stream = warp / (4 * kHalves), part = warp / 4 % kHalves, quarter = warp & 3, own = quarter * 32 + lane;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16, s_col = lanes + stream * 128, p_col = lanes + S::weights(stream), o_col = lanes + S::sums(stream);
        const uint32_t q_operand = q_at + stream * S::kOperand;
        const int copies = SPLIT ? a.copies : 1, rows_own = 128 / copies;
        const int row = SPLIT ? own & (rows_own - 1) : stream * 128 + own;       // of the piece
        const int chunks = 4 / (copies * kHalves), chunk0 = SPLIT ? own / rows_own * chunks : chunks * part;      // columns of 32 that this thread has
        registers_up<Form::kSoftmaxRegs>();
        uint32_t tiles_done = 0, keys_done = 0;
        // The halves of a row meet at a barrier of their two warps, with a number of each.  One barrier a meeting will do where between two meetings at the same place there is one at
        // another: factors at place 2, tiles at 0 and 1 in turn, sums at that of the next tile.
        auto meet = [&](float x, uint32_t place) {
            float* at = sh.meet[place];
            at[tid] = x;
            chunk_sync(2 + 4 * stream + quarter, 64);
            return at[tid ^ 128];
        };
        while (const ChunkPiece* p = reader.next()) {
            const int n = p->n, mine = SPLIT ? (n + 1 - stream) / 2 : n;                  // tiles of this stream
            ChunkRow r{-1e30f, 0.0f, a.factor};
            if (n > 0) {
                const int first_row = SPLIT ? quarter * 32 : stream * 128 + quarter * 32;
                auto query = [&](int k) -> const uint16_t* {
                    const int at = SPLIT ? (first_row + k) & (rows_own - 1) : first_row + k;
                    return at < p->rows ? a.Q + p->row(a, at) * D : nullptr;
                };
                // (a half has the factors of its 16 rows in the lanes that the other half's 16 leave)
                r.factor = chunk_queries<D, FMT, kHalves>(a, q_operand, lane, quarter * 32, part, query);
                if constexpr (kHalves == 2) {
                    const float others = meet(r.factor, 2);
                    if (lane / 16 != part) r.factor = others;
                }
                fence_proxy_async();
                tcgen05_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&sh.q_full[stream]));
            }
            for (int i = 0; i < mine; ++i) {
                const int slot = (SPLIT ? keys_done + 2 * i + stream : tiles_done) & 7;
                wait(sh.s_full[stream], tiles_done & 1);
                tcgen05_after_sync();
                const int2 info = sh.info[slot];
                if (!(info.y >> (2 + stream) & 1)) {
                    const ChunkMask mask{info.x, info.y, row < p->rows ? p->position(a, row) : -1, a.window, a.sinks};
                    chunk_hide(mask, s_col, chunk0, chunks);
                }
                auto ahead = [&] {
                    // the weights' place and the sums are free once the products of the tile before are done
                    wait(sh.o_full[stream], (tiles_done & 1) ^ 1);
                    tcgen05_after_sync();
                };
                auto same = [](float x) { return x; };
                const uint32_t read = smem_addr(&sh.s_free[stream]);
                if constexpr (!SPLIT && kHalves == 1) {
                    chunk_softmax<D, FMT, 4, false, D>(r, sh.scale[slot], s_col, p_col, 0, read, ahead, same, i > 0, o_col);
                } else if constexpr (!SPLIT) {
                    chunk_softmax<D, FMT, 2, false, D / 2>(r, sh.scale[slot], s_col, p_col, chunk0, read, ahead, [&](float x) { return fmaxf(x, meet(x, tiles_done & 1)); }, i > 0, o_col + part * (D / 2));
                } else {
                    if (copies == 1) chunk_softmax<D, FMT, 4, true, D>(r, sh.scale[slot], s_col, p_col, chunk0, read, ahead, same, i > 0, o_col);
                    else if (copies == 2) chunk_softmax<D, FMT, 2, false, D>(r, sh.scale[slot], s_col, p_col, chunk0, read, ahead, same, i > 0, o_col);
                    else chunk_softmax<D, FMT, 1, false, D>(r, sh.scale[slot], s_col, p_col, chunk0, read, ahead, same, i > 0, o_col);
                    if (!S::kApart || tiles_done == 0) {               // the weights of the other copies' keys; in a place of their own they stay zeros
                        uint32_t zero[16] = {};
#pragma unroll 1
                        for (int c = 0; c < 4; ++c)
                            if (c < chunk0 || c >= chunk0 + chunks) tmem_store(p_col + 16 * c, zero);
                    }
                }
                ++tiles_done;
                tmem_stored();
                tcgen05_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&sh.p_full[stream]));
            }
            keys_done += n;
            if (mine > 0) {
                wait(sh.o_full[stream], (tiles_done & 1) ^ 1);
                tcgen05_after_sync();
            }
            const float m = r.m;
            float l = r.l;
            if constexpr (!SPLIT) {
                if (wait.lost) l = __int_as_float(0x7fc00000);
                if (kHalves == 2 && n > 0) l += meet(l, tiles_done & 1);
            }
            // ---- the piece's sums
            float* slot = nullptr;
            if (p->place) slot = chunk_slot<D, SPLIT>(a, blockIdx.x, p->place);
            const bool there = row < p->rows;
            if constexpr (!SPLIT) {
                const float inv = l > 0.0f ? __fdiv_rn(1.0f, l) : l == 0.0f ? 0.0f : l;
                if (slot && there && part == 0) {
                    slot[kPerTile * D + row] = m;
                    slot[kPerTile * (D + 1) + row] = l;
                }
                uint16_t* out = there ? static_cast<uint16_t*>(a.O) + p->row(a, row) * D : nullptr;
#pragma unroll 1
                for (int c = part * (D / kHalves); c < (part + 1) * (D / kHalves); c += 32) {
                    uint32_t x[32] = {};
                    if (mine > 0) {
                        tmem_load(o_col + c, x);
                        tmem_loaded();
                    }
                    if (there && slot) {
#pragma unroll
                        for (int e = 0; e < 32; e += 4) *reinterpret_cast<uint4*>(slot + (size_t)row * D + c + e) = make_uint4(x[e], x[e + 1], x[e + 2], x[e + 3]);
                    } else if (there) {
                        if (FMT != FMT_FP4 && !a.bf16) {               // (4 bits: 61440 at most)
                            float top = 0.0f;
#pragma unroll
                            for (int e = 0; e < 32; e += 2) top = max3_abs(top, __uint_as_float(x[e]), __uint_as_float(x[e + 1]));
                            if (top * inv >= kChunkRoundsUp)
#pragma unroll
                                for (int e = 0; e < 32; ++e) x[e] = __float_as_uint(chunk_cut_down(__uint_as_float(x[e]), l));
                        }
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
                // The 2 x copies parts of every row meet in the queries' place: all channels at a time where the rows are few, else 16 of them.
                sh.m[tid] = m;
                __syncwarp();
                chunk_sync(1, 256);
                const int rows = p->rows, parts = 2 * copies;
                float* exchange = reinterpret_cast<float*>(rings);
                float most = -1e30f;
                for (int k = 0; k < parts; ++k) most = fmaxf(most, sh.m[k * rows_own + row]);
                const float r = ex2_approx(m - most);
                sh.l[tid] = wait.lost ? __int_as_float(0x7fc00000) : l * r;
                const bool wide = parts * rows * (D + 4) * 4 <= 2 * S::kOperand;
                const int width = wide ? D : 16, pitch = width + 4, quads = width / 4;
#pragma unroll 1
                for (int c0 = 0; c0 < D; c0 += width) {
                    auto put = [&](auto columns, int c) {
                        constexpr int C = decltype(columns)::value;
                        uint32_t x[C] = {};
                        if (mine > 0) {
                            tmem_load(o_col + c0 + c, x);
                            tmem_loaded();
                        }
                        if (there) {
                            float4* to = reinterpret_cast<float4*>(exchange + (tid / rows_own * rows + row) * pitch + c);
#pragma unroll
                            for (int e = 0; e < C / 4; ++e)
                                to[e] = make_float4(__uint_as_float(x[4 * e]) * r, __uint_as_float(x[4 * e + 1]) * r, __uint_as_float(x[4 * e + 2]) * r, __uint_as_float(x[4 * e + 3]) * r);
                        }
                        __syncwarp();
                    };
                    if (wide) {
#pragma unroll 1
                        for (int c = 0; c < D; c += 32) put(std::integral_constant<int, 32>(), c);
                    } else put(std::integral_constant<int, 16>(), 0);
                    chunk_sync(1, 256);
                    for (int i = tid; i < rows * quads; i += 256) {
                        const int at = i / quads, c = i % quads * 4;
                        float all = 0.0f;
                        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
                        for (int k = 0; k < parts; ++k) {
                            const float4 w = *reinterpret_cast<const float4*>(exchange + (k * rows + at) * pitch + c);
                            all += sh.l[k * rows_own + at];
                            v.x += w.x, v.y += w.y, v.z += w.z, v.w += w.w;
                        }
                        if (slot) {
                            *reinterpret_cast<float4*>(slot + (size_t)at * D + c0 + c) = v;
                            if (c0 + c == 0) slot[kPerTile * (D + 1) + at] = all;
                        } else {
                            *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.O) + p->row(a, at) * D + c0 + c) = chunk_out4(v, all, a.bf16);
                        }
                    }
                    if (slot && c0 == 0 && tid < rows) slot[kPerTile * D + tid] = most;      // (threads 0 .. rows - 1 are the first copies of their rows)
                    __syncwarp();
                    chunk_sync(1, 256);
                }
            }
            tcgen05_before_sync();
            reader.leave();
        }
        if (!a.merged) __threadfence();                                // as sa_rotate_qkv's kernel: a decode call behind this one reads its queries before it waits
    } else if (warp < kProducts) {
        // ---- operands: a key a thread (SPLIT: its key or its value, of every other tile)
        registers_down<Form::kOperandRegs>();
        const int part = warp & 3, row = part * 32 + lane;             // half page of the tile
        const int group = (warp - kOperands) >> 3;                     // SPLIT: which tiles
        const bool keys = !SPLIT || !(warp & 4), values = !SPLIT || (warp & 4);
        uint32_t keys_done = 0;
        while (const ChunkPiece* p = reader.next()) {
            const int n = p->n;
            for (int j = SPLIT ? (group ^ keys_done) & 1 : 0; j < n; j += SPLIT ? 2 : 1) {
                const uint32_t now = keys_done + j;
                const int stage = now % S::kStages, record = now % S::kRing, buffer = now % NB, slot = now & 7;
                // the operands' places are free once the products of the tile NB ahead are done: announced by turns at two barriers, so that warps which take every other tile have one
                const uint32_t free_at = now & 1, turn = ((now + 2 - NB) >> 1) - 1 & 1;
                wait(sh.raw_full[record], now / S::kRing & 1);
                const int2 info = sh.raw_info[stage];
                const uint8_t* half = raw + stage * S::kRaw + part * S::kHalf;
                // what no row sees is zero: it may hold anything, and a weight of zero times that is not zero
                bool seen = info.y >> 4 & 1;
                if (!seen) {
                    const int key = info.x + row;
                    seen = (info.y >> (part >> 1) & 1) && key < p->hi && (key >= p->lo || key < a.sinks);
                }
                if (keys) {
                    const uint32_t operand = k_at + buffer * S::kOperand;
                    ChunkCodes<D, FMT, true> codes(half, lane);
                    uint32_t scale = 0;
                    if constexpr (S::kScaled) scale = seen ? *reinterpret_cast<const uint16_t*>(half + S::kMeta + lane * 4) : 0u;
                    wait(sh.k_empty[free_at], turn);
                    // (of a key of zeros, whose scores are zeros, and of one that nobody sees: any number but zero, which -inf is multiplied by)
                    if constexpr (S::kScaled) sh.scale[slot][row] = scale ? half_bits_to_float(scale) : 1.0f;
                    if (row == 0) sh.info[slot] = info;
                    codes.put(half, lane, operand, row, seen);
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0 && !wait.lost) mbar_arrive(smem_addr(&sh.k_full[buffer]));
                }
                if (values) {
                    const uint32_t operand = v_at + buffer * S::kOperand;
                    ChunkCodes<D, FMT, false> codes(half, lane);
                    wait(sh.v_empty[free_at], turn);
                    codes.put(half, lane, operand, row, seen);
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0 && !wait.lost) mbar_arrive(smem_addr(&sh.v_full[buffer]));
                }
                if (lane == 0) mbar_arrive(smem_addr(&sh.raw_empty[record]));
            }
            keys_done += n;
            reader.leave();
        }
    } else if (warp == kProducts) {
        // ---- products
        registers_down<Form::kOtherRegs>();
        {
            const bool elected = elect_lane();
            const uint32_t q_first = smem_operand(q_at), k_first = smem_operand(k_at), v_first = smem_operand(v_at, 16384);
            constexpr uint32_t kScores = mma_form(kChunkTile, S::kBf16, false), kValues = mma_form(D, false, true);
            uint32_t keys_done = 0, pieces = 0, done[2] = {}, read[2] = {};          // of the streams: tiles whose values are issued, whose scores have been read
            auto scores = [&](int stream, uint32_t key_tile) {
                const uint32_t q = q_first + stream * (S::kOperand >> 4), k = k_first + key_tile % NB * (S::kOperand >> 4);
                const bool go = elected && !wait.lost;
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    const uint32_t off = ((i >> 2) * 16384 + (i & 3) * 32) >> 4;
                    tcgen05_mma_ss(stream * 128, q + off, k + off, kScores, i > 0, go);
                }
                if (go) mbar_arrive(smem_addr(&sh.s_full[stream]));
                tcgen05_commit(smem_addr(&sh.s_full[stream]), go);
            };
            auto commit = [&](const unsigned long long& bar) {
                tcgen05_commit(smem_addr(&bar), elected && !wait.lost);
            };
            auto values = [&](int stream, uint32_t key_tile, bool first) {
                const uint32_t v = v_first + key_tile % NB * (S::kOperand >> 4);
                wait(sh.p_full[stream], done[stream]++ & 1);
                tcgen05_after_sync();
                const bool go = elected && !wait.lost;
#pragma unroll
                for (int i = 0; i < kChunkTile / 16; ++i)
                    tcgen05_mma_ts(S::sums(stream), S::weights(stream) + 8 * i, v + i * 128, kValues, !first || i > 0, go);
                commit(sh.o_full[stream]);
            };
            auto key_ready = [&](uint32_t key_tile) {
                wait(sh.k_full[key_tile % NB], key_tile / NB & 1);
                tcgen05_after_sync();
            };
            auto scores_read = [&](int stream) {                       // (with the weights in their place that is known by the weights' being there)
                if constexpr (S::kApart) {
                    wait(sh.s_free[stream], read[stream]++ & 1);
                    tcgen05_after_sync();
                }
            };
            while (const ChunkPiece* p = reader.next()) {
                const int n = p->n;
                reader.leave();
                if (n == 0) continue;
                wait(sh.q_full[0], pieces & 1);
                const uint32_t g = keys_done;
                key_ready(g);
                scores(0, g);
                // (the first stream starts while the second still ends the piece before: 1 us of a prompt of 4096 tokens)
                wait(sh.q_full[1], pieces & 1);
                ++pieces;
                tcgen05_after_sync();
                if constexpr (!SPLIT) scores(1, g);
                commit(sh.k_empty[(g + NB) & 1]);
                if constexpr (SPLIT)
                    if (n > 1) {
                        key_ready(g + 1);
                        scores(1, g + 1);
                        commit(sh.k_empty[(g + 1 + NB) & 1]);
                    }
                for (int j = 0; j < n; ++j) {
                    const uint32_t now = g + j;
                    if constexpr (SPLIT && S::kApart) {
                        const int stream = j & 1;
                        scores_read(stream);
                        if (j + 2 < n) {
                            key_ready(now + 2);
                            scores(stream, now + 2);
                            commit(sh.k_empty[(now + 2 + NB) & 1]);
                        }
                        wait(sh.v_full[now % NB], now / NB & 1);
                        tcgen05_after_sync();
                        values(stream, now, j < 2);
                        commit(sh.v_empty[(now + NB) & 1]);
                    } else if constexpr (SPLIT) {
                        const int stream = j & 1;
                        wait(sh.v_full[now % NB], now / NB & 1);
                        tcgen05_after_sync();
                        values(stream, now, j < 2);
                        commit(sh.v_empty[(now + NB) & 1]);
                        scores_read(stream);
                        if (j + 2 < n) {
                            key_ready(now + 2);
                            scores(stream, now + 2);
                            commit(sh.k_empty[(now + 2 + NB) & 1]);
                        }
                    } else if constexpr (S::kApart) {
                        scores_read(0);
                        if (j + 1 < n) {
                            key_ready(now + 1);
                            scores(0, now + 1);
                        }
                        scores_read(1);
                        if (j + 1 < n) {
                            scores(1, now + 1);
                            commit(sh.k_empty[(now + 1 + NB) & 1]);
                        }
                        wait(sh.v_full[now % NB], now / NB & 1);
                        tcgen05_after_sync();
                        values(0, now, j == 0);
                        values(1, now, j == 0);
                        commit(sh.v_empty[(now + NB) & 1]);
                    } else {
                        wait(sh.v_full[now % NB], now / NB & 1);
                        tcgen05_after_sync();
                        values(0, now, j == 0);
                        if (j + 1 < n) {
                            key_ready(now + 1);
                            scores(0, now + 1);
                        }
                        values(1, now, j == 0);
                        commit(sh.v_empty[(now + NB) & 1]);
                        if (j + 1 < n) {
                            scores(1, now + 1);
                            commit(sh.k_empty[(now + 1 + NB) & 1]);
                        }
                    }
                }
                keys_done += n;
            }
            ChunkWait<1, LOST> end;                                           // (products in flight, also where a wait was lost)
            tcgen05_commit(smem_addr(&sh.done), elected);
            end(sh.done, 0);
        }
    } else if (warp == kProducts + 1) {
        // ---- loader
        registers_down<Form::kOtherRegs>();
        fence_proxy_async_global();                                    // (the records were written by ordinary stores)
        uint32_t keys_done = 0, copied = 0;
        while (const ChunkPiece* p = reader.next()) {
            const int n = p->n, hi = p->hi, head = p->head;
            const int32_t* table = a.c.page_table + (size_t)p->b * a.c.max_pages;
            for (int j0 = 0; j0 < n; j0 += 16) {                       // 16 tiles, two lanes a tile: a page and a stream each
                const int t0 = p->tile(min(j0 + lane / 2, n - 1)) * kChunkTile, page = t0 / kPageTokens + lane % 2;
                int at = -1;                                           // (none)
                if (j0 + lane / 2 < n && page < a.c.max_pages && page * kPageTokens < hi) at = table[page];
                if (at >= a.c.n_pages) at = -1;
                const uint32_t there = __ballot_sync(0xffffffffu, at >= 0);
                const bool both = (there >> (lane & 30) & 3) == 3;
                const uint32_t whole = __ballot_sync(0xffffffffu, both && p->first[lane % 2] - t0 >= kChunkTile - 1 && (a.window == 0 || p->last[lane % 2] - t0 < a.window || t0 + kChunkTile <= a.sinks));
                const uint32_t seen = __ballot_sync(0xffffffffu, both && hi - t0 >= kChunkTile && (t0 >= p->lo || t0 + kChunkTile <= a.sinks));
                for (int i = 0; i < 16 && j0 + i < n; ++i, ++keys_done) {
                    const int at0 = __shfl_sync(0xffffffffu, at, 2 * i), at1 = __shfl_sync(0xffffffffu, at, 2 * i + 1), first = __shfl_sync(0xffffffffu, t0, 2 * i);
                    const uint32_t stage = keys_done % S::kStages, before = keys_done - S::kStages;      // (before: the tile whose place this one takes)
                    if (keys_done >= (uint32_t)S::kStages) wait(sh.raw_empty[before % S::kRing], before / S::kRing & 1);
                    const bool never = LOST && first == a.lost_tile * kChunkTile && p->b == a.lost_b && head == a.lost_head;
                    if (lane == 0 && !wait.lost && !never) {
                        const uint32_t bar = smem_addr(&sh.raw_full[keys_done % S::kRing]), to = smem_addr(raw + stage * S::kRaw);
                        sh.raw_info[stage] = make_int2(first, (there >> 2 * i & 3) | (whole >> 2 * i & 3) << 2 | (seen >> 2 * i & 1) << 4);
                        mbar_arrive_expect_tx(bar, ((at0 >= 0) + (at1 >= 0)) * 2u * S::kHalf);
                        if (at0 >= 0) bulk_g2s(to, a.c.pages + ((size_t)at0 * a.c.Hkv + head) * (2 * S::kHalf), 2 * S::kHalf, bar);
                        if (at1 >= 0) bulk_g2s(to + 2 * S::kHalf, a.c.pages + ((size_t)at1 * a.c.Hkv + head) * (2 * S::kHalf), 2 * S::kHalf, bar);
                    }
                    __syncwarp();
                    copied += !wait.lost;
                }
            }
            reader.leave();
        }
        copied = __shfl_sync(0xffffffffu, copied, 0);
        // copies in flight land before the block ends, also where the operands' warps have given up
        const uint32_t last = copied < (uint32_t)S::kStages ? copied : (uint32_t)S::kStages;
        for (uint32_t i = 0; i < last; ++i) {
            const uint32_t k = copied - 1 - i;
            ChunkWait<1, LOST> landed;
            landed(sh.raw_full[k % S::kRing], k / S::kRing & 1);
        }
    } else if (warp == kProducts + 2) {
        // ---- the deal: the block's stretch of all units' tiles, piece by piece
        registers_down<Form::kOtherRegs>();
        for (int i = lane; i < a.s.n; i += 32) sh.lens[i] = max(a.c.seq_lens[a.s.b[i]], 0);
        __syncwarp();
        const int n_flat = a.s.tiles[a.s.n];
        int head, flat, skip = 0;                                      // the unit, and how far into it (its fixed cost included) the stretch starts
        uint64_t at = 0, end_at = 1, per = 1;                          // the stretch; the length of one
        bool whole = a.whole;
        if (!whole) {
            const int each = (n_flat + 31) / 32, mine0 = min(lane * each, n_flat), mine1 = min(mine0 + each, n_flat);
            uint64_t cost = 0;
            uint32_t longest = 0;
            for (int i = mine0; i < mine1; ++i) {
                const uint32_t c = kChunkUnitCost + chunk_unit(a, sh.lens, i, per_tile).count;
                cost += c;
                longest = max(longest, c);
            }
            longest = __reduce_max_sync(0xffffffffu, longest);
            uint64_t ahead = cost;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint64_t x = __shfl_up_sync(0xffffffffu, ahead, o);
                if (lane >= o) ahead += x;
            }
            const uint64_t sum = __shfl_sync(0xffffffffu, ahead, 31), total = sum * a.c.Hkv;
            ahead -= cost;
            // equal stretches but for the last; 32-bit divisions where the numbers allow (64-bit ones are long routines)
            per = total >> 32 == 0 ? ((uint32_t)total - 1) / gridDim.x + 1 : (total - 1) / gridDim.x + 1;
            // A unit a block where the longest costs no more than an equal stretch and what cutting costs.
            whole = (uint64_t)n_flat * a.c.Hkv <= gridDim.x && longest <= per + chunk_cut_cost(D, SPLIT);
            at = min(per * blockIdx.x, total);
            end_at = min(at + per, total);
            head = (int)(total >> 32 == 0 ? (uint32_t)at / (uint32_t)sum : at / sum);
            uint64_t rest = at - head * sum;
            const uint32_t owner = __ballot_sync(0xffffffffu, rest >= ahead && rest - ahead < cost);      // the lane that has the unit at which the stretch starts (none: no stretch)
            int i = mine0;
            if (owner >> lane & 1u)
                for (rest -= ahead;; ++i) {
                    const uint32_t c = kChunkUnitCost + chunk_unit(a, sh.lens, i, per_tile).count;
                    if (rest < c) break;
                    rest -= c;
                }
            const int from = owner ? __ffs(owner) - 1 : 0;
            flat = __shfl_sync(0xffffffffu, i, from);
            skip = (int)__shfl_sync(0xffffffffu, (uint32_t)rest, from);
        }
        if (whole) {
            head = blockIdx.x / n_flat;
            flat = blockIdx.x % n_flat;
            at = skip = 0;
            end_at = head < a.c.Hkv;
        }
        uint32_t made = 0;
        bool cut = false;
        ChunkWait<16, LOST> free;
        bool lost = false;                                             // no place came free: nothing more is handed out
        auto place = [&]() -> ChunkPiece& {
            free(sh.piece_empty[made % kChunkPieces], made / kChunkPieces & 1 ^ 1);
            lost = __any_sync(0xffffffffu, free.lost) || (LOST && a.lost_tile < 0 && (int)made >= -1 - a.lost_tile);
            return sh.pieces[made % kChunkPieces];
        };
        auto ready = [&] {
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&sh.piece_full[made % kChunkPieces]));
            ++made;
        };
        auto deal = [&](auto whether) {
            constexpr bool handed_out = decltype(whether)::value;
            while (at < end_at) {
                const ChunkUnit u = chunk_unit(a, sh.lens, flat, per_tile);
                const int cost = kChunkUnitCost + u.count, to = whole || end_at - at >= (uint64_t)(cost - skip) ? cost : skip + (int)(end_at - at);
                const int begin = max(skip - kChunkUnitCost, 0), end = max(to - kChunkUnitCost, 0);
                if (end > begin || (u.count == 0 && skip == 0)) {
                    ChunkPiece& p = handed_out ? place() : sh.undealt;
                    if (handed_out && lost) return;
                    if (lane == 0) {
                        const int token = a.by_group(u.row0);
                        p.n = end - begin;
                        p.head = head;
                        p.b = a.s.b[u.seq];
                        p.rows = u.rows;
                        p.token_row = u.row0 - token * a.G;
                        p.token = u.first;
                        p.q_token = a.s.row0[u.seq] + token;
                        p.lo = u.lo;
                        p.hi = u.hi;
                        p.sink_tiles = u.sink_tiles;
                        p.window_tile = u.window_tile;
                        p.begin = begin;
                        p.place = begin == 0 && end == u.count ? 0 : begin == 0 ? 2 : 1;
                        if (p.place == 2) {
                            const uint64_t last = at - skip + cost - 1;    // where the unit's last tile is
                            p.last_block = (int)(last >> 32 == 0 ? (uint32_t)last / (uint32_t)per : last / per);
                        }
                        for (int i = 0; i < 2; ++i) {
                            p.first[i] = p.position(a, SPLIT ? 0 : min(i * 128, u.rows - 1));
                            p.last[i] = p.position(a, SPLIT ? u.rows - 1 : min(i * 128 + 127, u.rows - 1));
                        }
                        if (p.place == 2) {
                            *chunk_cut(a, blockIdx.x) = p;
                            cut = true;
                        }
                    }
                    if (handed_out) {
                        ready();
                    } else {
                        __syncwarp();
                        chunk_undealt<D, SPLIT>(a, p, lane);
                        __syncwarp();
                    }
                }
                at += whole ? 1 : to - skip;
                skip = 0;
                if (++flat == n_flat) flat = 0, ++head;
            }
        };
        deal(std::true_type());
        if (lost) deal(std::false_type());
        if (lane == 0 && !cut) chunk_cut(a, blockIdx.x)->place = 0;
        if (!lost) {
            ChunkPiece& p = place();
            if (!lost) {
                if (lane == 0) p.n = -1;
                ready();
            }
        }
    } else {
        registers_down<Form::kOtherRegs>();
    }
    tcgen05_before_sync();
    __syncthreads();
    tcgen05_after_sync();
    if (warp == kProducts) tmem_free();
}

// Units that the deal has cut: block (x, y) takes ROWS rows of the one that starts in block x of the kernel above.  Its threads are dealt to 4 channels of a row each, and where
// there are more of them to the parts, of which an order independent of time is kept.
template <int D, bool SPLIT>
SA_HD constexpr int chunk_merge_rows() { return (SPLIT ? 256 : 2048) / D; }
template <int D, bool SPLIT>
__global__ void __launch_bounds__(256) chunk_merge_kernel(const __grid_constant__ ChunkArgs a) {
    constexpr int kPerTile = chunk_rows(SPLIT), kRows = chunk_merge_rows<D, SPLIT>(), kQuads = D / 4, kItems = kRows * kQuads, kGroups = kItems < 256 ? 256 / kItems : 1, kLanes = 256 / kRows;
    constexpr size_t kSlot = chunk_slot_floats(D, SPLIT);
    static_assert(kItems % 256 == 0 || 256 % kItems == 0, "items are dealt evenly");
    __shared__ float meet[2][256];
    __shared__ float4 sums[kGroups > 1 ? 256 : 1];
    pdl_wait();
    const ChunkPiece& p = *chunk_cut(a, blockIdx.x);
    const int tid = threadIdx.x, row0 = blockIdx.y * kRows, first = blockIdx.x;
    if (p.place != 2 || row0 >= p.rows) return;
    const int rows = p.rows, last = p.last_block;
    const float* slots = reinterpret_cast<const float*>(a.workspace + kChunkCutBytes);
    auto part = [&](int k) { return slots + (size_t)(k == first ? 2 * k + 1 : 2 * k) * kSlot; };
    // references and sums of the rows: kLanes threads a row
    const int at = tid / kLanes, row = min(row0 + at, rows - 1);
    auto all_lanes = [&](float x, int place, auto join) {
        meet[place][tid] = x;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kLanes; ++k) x = k ? join(x, meet[place][at * kLanes + k]) : meet[place][at * kLanes];
        return x;
    };
    float most = -1e30f, l = 0.0f;
    for (int k = first + tid % kLanes; k <= last; k += kLanes) most = fmaxf(most, part(k)[kPerTile * D + row]);
    most = all_lanes(most, 0, [](float x, float y) { return fmaxf(x, y); });
    for (int k = first + tid % kLanes; k <= last; k += kLanes) l += part(k)[kPerTile * (D + 1) + row] * ex2_approx(part(k)[kPerTile * D + row] - most);
    l = all_lanes(l, 1, [](float x, float y) { return x + y; });
    __syncthreads();
    meet[0][tid] = most;
    meet[1][tid] = l;
    __syncthreads();
    for (int i = tid; i < kItems * kGroups; i += 256) {
        const int item = i % kItems, group = i / kItems, r = item / kQuads, c = item % kQuads * 4;
        const bool there = row0 + r < rows;
        const float top = meet[0][r * kLanes], all = meet[1][r * kLanes];
        float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (there)
#pragma unroll 4
            for (int k = first + group; k <= last; k += kGroups) {
                const float* s = part(k);
                const float f = ex2_approx(s[kPerTile * D + row0 + r] - top);
                const float4 x = *reinterpret_cast<const float4*>(s + (size_t)(row0 + r) * D + c);
                o.x += x.x * f, o.y += x.y * f, o.z += x.z * f, o.w += x.w * f;
            }
        if constexpr (kGroups > 1) {
            sums[tid] = o;
            __syncthreads();
            if (group == 0)
#pragma unroll
                for (int k = 1; k < kGroups; ++k) {
                    const float4 x = sums[tid + k * kItems];
                    o.x += x.x, o.y += x.y, o.z += x.z, o.w += x.w;
                }
        }
        if (there && group == 0) *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.O) + p.row(a, row0 + r) * D + c) = chunk_out4(o, all, a.bf16);
    }
    __threadfence();
}

template <int D, int FMT, bool SPLIT, bool LOST = false>
cudaError_t launch_chunk(const ChunkArgs& a, int blocks, int rows_most, cudaStream_t s) {
    static OncePerDevice once;
    if (!allow_shared(chunk_kernel<D, FMT, SPLIT, LOST>, ChunkShape<D, FMT>::kBytes, once)) return cudaGetLastError();
    const cudaError_t e = launch_pdl(chunk_kernel<D, FMT, SPLIT, LOST>, dim3(blocks), dim3(ChunkForm<D, SPLIT>::kThreads), (size_t)ChunkShape<D, FMT>::kBytes, s, a);
    if (e != cudaSuccess || !a.merged) return e;
    return launch_pdl(chunk_merge_kernel<D, SPLIT>, dim3(blocks, (rows_most - 1) / chunk_merge_rows<D, SPLIT>() + 1), dim3(256), 0, s, a);
}

cudaError_t launch_chunk_pot(int d, int fmt, bool split, const ChunkArgs& a, int blocks, int rows_most, cudaStream_t s);
cudaError_t launch_chunk_plain(int d, int fmt, bool split, const ChunkArgs& a, int blocks, int rows_most, cudaStream_t s);
cudaError_t launch_chunk_lost(bool split, const ChunkArgs& a, int blocks, int rows_most, cudaStream_t s);      // (sa_chunk_pot.cu; head_dim 64, PoT-M4 in bytes)

}  // namespace sa
