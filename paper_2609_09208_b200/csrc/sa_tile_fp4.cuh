// Attention of one query group over one staged tile of the 4-bit cache: 64 keys (a page) at head_dim 64, 32 at 128.
//
// The state and its merge are those of TileMma; the numbers are plain binary16 (a code times its scale, exact), so there is no scale in a
// logit or a weight, and a weight is w = 2^(z - R + 14), in two binary16 terms (22 significant bits, sa_tile_mma.cuh).
// A block of at most 4 queries (kPair) puts both terms into one product: the products have 8 columns, queries n and n + 4 are the same
// one, and the first term of its weights goes to column n, the second to column n + 4: half the products of A.V (head_dim 128, 32 / 8
// heads, 16 x 8192 tokens: 41.0 -> 36.5 us).
//
// What a tile costs is issue slots (for 32 keys of head_dim 64 and 8 queries: 64 conversions and 64 packed products of codes and scales, 24 matrix
// products, 50 for the softmax), on pipes that are each about half full; hence
//   * 64 keys at a time at head_dim 64: the loop around a tile, its vote and its sums are paid for once (32 x 32 768 tokens 79.4 -> 72.7 us);
//   * value scales decoded once per warp: eight lanes need each of them;
//   * the way of the rare tiles (the first ones, a reference that moves, slots past the sequence's end) has its own copy of what follows:
//     joined behind the softmax it cost every tile 20 moves;
//   * what the first term leaves of a weight by FP32 fma with a binary16 operand (full rate; a conversion takes two slots).
#pragma once
#include "sa_tile_mma.cuh"

namespace sa {

template <int D, int FMT, bool LONG, bool FINE>
struct TileFp4 : TileMma<D, FMT, LONG, FINE> {
    using Base = TileMma<D, FMT, LONG, FINE>;
    using Stage = typename Base::Stage;
    using Base::acc, Base::l, Base::nR, Base::plain, Base::q, Base::qs, Base::seen, Base::kPair, Base::MT;
    static constexpr int NJ = 4 * Stage::kHalves;  // groups of 8 keys
    static constexpr int kScratchBytes = Stage::kHalves * 4 * D;
    uint32_t scratch;                              // shared address of this warp's decoded value scales

    SA_D void tile(const DecodeArgs& a, uint32_t st, int n_valid, int lane, int, int, int) {
        value_scales<false>(st, a.one, lane, 0);
        float z[NJ][2], none[1][2];
#pragma unroll
        for (int hf = 0; hf < Stage::kHalves; ++hf) {
            const uint32_t at = st + hf * Stage::kHalfBytes;
            q.tile(at, at + Stage::kPlaneOff, lane, a.one, *reinterpret_cast<float(*)[4][2]>(&z[4 * hf]), none);
        }
        float w[NJ][2];
        __half2 h[NJ];
        if (LONG && __builtin_expect(n_valid >= plain, 1)) {
            if (__builtin_expect(!__any_sync(0xffffffffu, weights(z, w, h)), 1)) {
                finish(st, w, h, lane);
                return;
            }
        }
        rare(z, w, h, a, st, n_valid, lane);
        finish(st, w, h, lane);
    }

private:
    // Weights of the tile and their first terms; whether one is beyond binary16: it has become infinite, 0x7c00, the only value that 0x0400
    // carries into the sign bit.
    SA_D bool weights(const float (&z)[NJ][2], float (&w)[NJ][2], __half2 (&h)[NJ]) const {
        const f32x2 from = add2(nR, pack_f32x2((float)kWeightShift, (float)kWeightShift));
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            float x0, x1;
            unpack_f32x2(ffma2(pack_f32x2(z[j][0], z[j][1]), qs, from), &x0, &x1);
            w[j][0] = ex2_approx(x0);
            w[j][1] = ex2_approx(x1);
        }
        return round_weights(w, h);
    }
    SA_D static bool round_weights(const float (&w)[NJ][2], __half2 (&h)[NJ]) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) h[j] = __floats2half2_rn(w[j][0], w[j][1]);
        __half2 top = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
        if constexpr (NJ == 8) top = __hmax2(top, __hmax2(__hmax2(h[4], h[5]), __hmax2(h[6], h[7])));
        return ((*reinterpret_cast<const uint32_t*>(&top) + 0x04000400u) & 0x80008000u) != 0u;
    }
    // The same for a first tile, one whose weights do not fit, and one with slots past the sequence's end, which may hold anything.
    SA_D void rare(const float (&z)[NJ][2], float (&w)[NJ][2], __half2 (&h)[NJ], const DecodeArgs& a, uint32_t st, int n_valid, int lane) {
        const int r = lane >> 2;
        bool move = !seen;                                    // warp-uniform
        for (int turn = 0; turn < 2; ++turn) {                // (a reference that has moved fits)
            if (move) {
                float s0, s1, y0 = -INFINITY, y1 = -INFINITY; // largest z of the tile, not rounded down
                unpack_f32x2(qs, &s0, &s1);
#pragma unroll
                for (int j = 0; j < NJ; ++j)
                    if (8 * j + r < n_valid) {
                        y0 = fmaxf(y0, __fmul_ru(z[j][0], s0));
                        y1 = fmaxf(y1, __fmul_ru(z[j][1], s1));
                    }
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) {
                    y0 = fmaxf(y0, __shfl_xor_sync(0xffffffffu, y0, o));
                    y1 = fmaxf(y1, __shfl_xor_sync(0xffffffffu, y1, o));
                }
                y0 = fminf(fmaxf(ceilf(y0), -kRefMax), kRefMax);
                y1 = fminf(fmaxf(ceilf(y1), -kRefMax), kRefMax);
                if (seen) {
                    float nR0, nR1;
                    unpack_f32x2(nR, &nR0, &nR1);
                    y0 = fmaxf(-nR0, y0);
                    y1 = fmaxf(-nR1, y1);
                    const float f0 = pow2i_neg(__float2int_rn(-nR0 - y0)), f1 = pow2i_neg(__float2int_rn(-nR1 - y1));
                    l = mul2(l, pack_f32x2(f0, f1));
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        acc[mt][0] *= f0;
                        acc[mt][1] *= f1;
                        acc[mt][2] *= f0;
                        acc[mt][3] *= f1;
                    }
                }
                nR = pack_f32x2(-y0, -y1);
                seen = true;
                plain = Stage::kTokens;
            }
            weights(z, w, h);
            if (n_valid < Stage::kTokens) {
#pragma unroll
                for (int j = 0; j < NJ; ++j)
                    if (8 * j + r >= n_valid) w[j][0] = w[j][1] = 0.0f;
                value_scales<true>(st, a.one, lane, n_valid); // scales may be NaN, and 0 * NaN is not 0
            }
            move = __any_sync(0xffffffffu, round_weights(w, h));
            if (__builtin_expect(!move, 1)) break;
        }
    }
    // Normaliser, second terms, A.V.
    SA_D void finish(uint32_t st, const float (&w)[NJ][2], const __half2 (&h)[NJ], int lane) {
        const int c = lane & 3;
        uint32_t bh[NJ], bl[kPair ? 1 : NJ];                  // operand fragments: keys 8 j + 2 c, + 1 of query r
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const uint32_t hi = *reinterpret_cast<const uint32_t*>(&h[j]);
            l = add2(l, pack_f32x2(w[j][0], w[j][1]));
            float x0, x1;                                     // what the first term leaves
            floats_minus_half2(w[j][0], w[j][1], hi, &x0, &x1);
            const __half2 rest = __floats2half2_rn(x0, x1);
            const uint32_t lo = *reinterpret_cast<const uint32_t*>(&rest);
            if constexpr (kPair) bh[j] = movmatrix_trans(c < 2 ? hi : lo);
            else {
                bh[j] = movmatrix_trans(hi);
                bl[j] = movmatrix_trans(lo);
            }
        }
        // 16 bytes of a lane are the codes of 32 dims (two row tiles) and all its keys of 32
#pragma unroll
        for (int g = 0; g < MT / 2; ++g) {
            float own[2][4];                                  // FINE: the sums of this tile
#pragma unroll
            for (int hf = 0; hf < Stage::kHalves; ++hf) {
                uint32_t codes[4], scales[2][4];              // scales: [row tile][tokens % 32 / 8]
                lds_u32x4(codes, st + hf * Stage::kHalfBytes + Stage::kVOff + g * 512 + lane * 16);
                lds_u32x4(scales[0], scratch + hf * 4 * D + g * 128 + c * 16);
                lds_u32x4(scales[1], scratch + hf * 4 * D + g * 128 + 64 + c * 16);
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    float(&sum)[4] = FINE ? own[m] : acc[2 * g + m];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        uint32_t v[4];
                        const uint32_t s0 = scales[m][2 * k], s1 = scales[m][2 * k + 1];
                        const int j = 4 * hf + 2 * k;
                        fp4_to_half2(codes[2 * m + k], v);
                        v[0] = mul_half2(v[0], s0);
                        v[1] = mul_half2(v[1], s0);
                        v[2] = mul_half2(v[2], s1);
                        v[3] = mul_half2(v[3], s1);
                        if (FINE && j == 0) mma_f16_16816_first(sum, v[0], v[1], v[2], v[3], bh[0], bh[1]);
                        else mma_f16_16816(sum, v[0], v[1], v[2], v[3], bh[j], bh[j + 1]);
                        if constexpr (!kPair) mma_f16_16816(sum, v[0], v[1], v[2], v[3], bl[j], bl[j + 1]);
                    }
                }
            }
            if constexpr (FINE) {
                add_sums(acc[2 * g], own[0]);
                add_sums(acc[2 * g + 1], own[1]);
            }
        }
    }
    SA_D static void add_sums(float (&to)[4], const float (&x)[4]) {
        unpack_f32x2(add2(pack_f32x2(to[0], to[1]), pack_f32x2(x[0], x[1])), &to[0], &to[1]);
        unpack_f32x2(add2(pack_f32x2(to[2], to[3]), pack_f32x2(x[2], x[3])), &to[2], &to[3]);
    }
    // Which of the keys `key`, key + 1 count, as a mask of a pair of binary16.
    SA_D static uint32_t keep_pair(int key, int n_valid) { return key >= n_valid ? 0u : key + 1 >= n_valid ? 0x0000ffffu : 0xffffffffu; }
    // The tile's value scales as binary16 pairs (two tokens of a block) into the warp's scratch, [half][d / 16][c][tokens % 32 / 8].
    // MASKED: 0 for slots past the sequence's end.
    template <bool MASKED>
    SA_D void value_scales(uint32_t st, uint32_t one, int lane, int n_valid) const {
        if (MASKED) __syncwarp();
#pragma unroll
        for (int i = 0; i < Stage::kHalves * D / 64; ++i) {
            const int hf = i / (D / 64), w = i % (D / 64) * 32 + lane;            // word w: [d / 32][c][row tile][k]
            const uint32_t x = lds_u32(st + hf * Stage::kHalfBytes + Stage::kVOff + 16 * D + w * 4);
            uint32_t s0 = fp4_pair_scale0(x, one), s1 = fp4_pair_scale1(x, one);
            if (MASKED) {
                const int key = 32 * hf + 16 * (w & 1) + 2 * (w >> 2 & 3);
                s0 &= keep_pair(key, n_valid);
                s1 &= keep_pair(key + 8, n_valid);
            }
            sts_u32x2(scratch + hf * 4 * D + (w >> 4) * 128 + (w >> 1 & 1) * 64 + (w >> 2 & 3) * 16 + (w & 1) * 8, s0, s1);
        }
        __syncwarp();
    }
};

// What a warp does with its tiles.
template <int D, int FMT, bool LONG, bool FINE, bool FP4 = format_fp4(FMT)>
struct TileOf {
    using type = TileMma<D, FMT, LONG, FINE>;
};
template <int D, int FMT, bool LONG, bool FINE>
struct TileOf<D, FMT, LONG, FINE, true> {
    using type = TileFp4<D, FMT, LONG, FINE>;
};
template <int D, int FMT, bool LONG, bool FINE>
using Tile = typename TileOf<D, FMT, LONG, FINE>::type;

}  // namespace sa
