// The 4-bit cache (SA_KV_FP4): number format, and the order of the codes in half a page block.
//
// A vector of d channels is cut into blocks of 16.  A block's scale is s = max|x| / 6 rounded to an unsigned 8-bit float (5 bits of
// exponent, 3 of mantissa: a binary16 pattern without its sign and its lowest 7 bits), at most 10240; a channel's code is x / s
// rounded to the nearest of +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} (ties to the even code, at most 6).  Both decisions are those of the
// exact quotients: a binary16 number over 6, or over a scale of 4 bits, is a tie or at least 2^-11 (relative) from one.
// A code times its scale has 6 significant bits and is a binary16 number, so the products of the attention start from exact operands.
//
// Half a block, 32 tokens (t: token in it, c: channel), is laid out for the lanes of the matrix products, r = lane / 4, q = lane % 4:
//   key codes     chunk k = 2 (c / 64) + c / 8 % 2 of 16 bytes a token at (32 k + t) 16; its word c / 16 % 4 holds 8 channels, two a byte.
//                 One ldmatrix gives a lane word q of tokens r, r + 8, r + 16, r + 24: all its channels are of block q, one scale;
//   key scales    [c / 64][c / 16 % 4][t % 8][t / 8]: the scales of a lane's four tokens are one word;
//   value codes   [c / 32][c % 8][t % 8 / 2][c / 16 % 2][t / 16][t / 8 % 2][c / 8 % 2], a byte: tokens t, t + 1 (t even) of one channel, the
//                 pair that a register of the transposed operand holds.  16 bytes of a lane are all it needs of 32 channels;
//   value scales  [c / 32][t % 8 / 2][c / 16 % 2][t / 16][t % 2][t / 8 % 2]: of a word, bytes 0, 2 and 1, 3 scale two pairs of tokens.
#pragma once
#include "sa_common.cuh"
#include "sa_quant.cuh"

namespace sa {

constexpr uint32_t kFp4ScaleMost = 0xe2u;              // 10240: 6 times that is the largest below 65504
constexpr uint32_t kFp4ScaleNaN = 0xffu;

// x / s, correctly rounded where it matters (see above): exact for quotients of a few bits, within an ulp otherwise.
SA_HD float fp4_quotient(float x, float s, float inv) {
    const float r = x * inv;
#ifdef __CUDA_ARCH__
    return __fmaf_rn(__fmaf_rn(-r, s, x), inv, r);
#else
    return fmaf(fmaf(-r, s, x), inv, r);
#endif
}
// 1 / s within two units in the last place, which the step of fp4_quotient makes good; 0 for 0.
SA_D float fp4_inverse(float s) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
    return s > 0.0f ? r : 0.0f;
}
// Scale byte of a block whose largest magnitude has the binary16 bits `amax`.  An infinity or NaN marks the whole block: NaN.
SA_D uint32_t fp4_scale_byte(uint32_t amax) {
    const float t = fp4_quotient(half_bits_to_float(amax), 6.0f, 1.0f / 6.0f);
    const uint32_t u = __float_as_uint(t);
    const uint32_t normal = ((u + 0x7ffffu + ((u >> 20) & 1u)) >> 20) - (112u << 3);
    const uint32_t b = t >= 0x1p-14f ? normal : (uint32_t)__float2int_rn(t * 0x1p17f);
    return amax < 0x7c00u ? min(b, kFp4ScaleMost) : kFp4ScaleNaN;
}
SA_D float fp4_scale(uint32_t byte) { return half_bits_to_float(byte << 7); }
// Codes of 8 channels (pairs of binary16), the first in the lowest nibble.  The quotients as fp4_quotient's, two at a time.
SA_D uint32_t fp4_codes(const uint32_t (&x)[4], float s, float inv) {
    float q[8];
    const f32x2 minus = pack_f32x2(-s, -s), i2 = pack_f32x2(inv, inv);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&x[i]));
        const f32x2 v = pack_f32x2(f.x, f.y), r = mul2(v, i2);
        unpack_f32x2(ffma2(ffma2(r, minus, v), i2, r), &q[2 * i], &q[2 * i + 1]);
    }
    uint32_t w;
    asm("{.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\tmov.b32 %0, {a, b, c, d};}"
        : "=r"(w)
        : "f"(q[0]), "f"(q[1]), "f"(q[2]), "f"(q[3]), "f"(q[4]), "f"(q[5]), "f"(q[6]), "f"(q[7]));
    return w;
}
// A block of 16 channels (pairs of binary16): codes of 8 and 8 channels; returns its scale byte.
SA_D uint32_t fp4_block(const uint32_t (&x)[8], uint32_t (&w)[2]) {
    uint32_t top = x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) asm("max.NaN.xorsign.abs.f16x2 %0, %0, %1;" : "+r"(top) : "r"(x[i]));      // two magnitudes at a time, with signs that do not matter
    const uint32_t b = fp4_scale_byte(max(top & 0x7fffu, (top >> 16) & 0x7fffu));
    const float s = fp4_scale(b), inv = fp4_inverse(s);
    const uint32_t lo[4] = {x[0], x[1], x[2], x[3]}, hi[4] = {x[4], x[5], x[6], x[7]};
    w[0] = fp4_codes(lo, s, inv);
    w[1] = fp4_codes(hi, s, inv);
    return b;
}
// The 8 codes of a word as pairs of binary16.
SA_D void fp4_to_half2(uint32_t w, uint32_t (&h)[4]) {
    asm("{.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\tcvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(w));
}
SA_D uint32_t mul_half2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
// Two floats minus a pair of binary16, exactly where they round to it.
SA_D void floats_minus_half2(float x, float y, uint32_t h, float* dx, float* dy) {
    asm("{.reg .b16 l, h, m;\n\tmov.b32 {l, h}, %2;\n\tmov.b16 m, 0xbc00;\n\tfma.rn.f32.f16 %0, l, m, %3;\n\tfma.rn.f32.f16 %1, h, m, %4;}" : "=f"(*dx), "=f"(*dy) : "r"(h), "f"(x), "f"(y));
}
// Byte J of a word of scales, twice, as binary16 (one: the value 1, opaque: a shift as a multiplication).
template <int J>
SA_D uint32_t fp4_scale2(uint32_t w, uint32_t one) {
    return __byte_perm(w, 0u, 0x4040u + 0x0101u * J) * (one * 128u);
}
// Scales of the two pairs of tokens of a word of value scales.
SA_D uint32_t fp4_pair_scale0(uint32_t w, uint32_t one) { return (w & 0x00ff00ffu) * (one * 128u); }
SA_D uint32_t fp4_pair_scale1(uint32_t w, uint32_t one) { return __byte_perm(w, 0u, 0x4341u) * (one * 128u); }

// Places in half a block, from the start of the key codes (first two) or of the value codes.
SA_HD int fp4_key_byte(int t, int c) { return (2 * (c / 64) + c / 8 % 2) * 512 + t * 16 + c / 16 % 4 * 4 + c % 8 / 2; }
SA_HD int fp4_key_scale(int d, int t, int c) { return 16 * d + c / 64 * 128 + c / 16 % 4 * 32 + t % 8 * 4 + t / 8; }
SA_HD int fp4_value_byte(int t, int c) {
    return c / 32 * 512 + c % 8 * 64 + t % 8 / 2 * 16 + c / 16 % 2 * 8 + t / 16 * 4 + t / 8 % 2 * 2 + c / 8 % 2;
}
SA_HD int fp4_value_scale(int d, int t, int c) { return 16 * d + c / 32 * 64 + t % 8 / 2 * 16 + c / 16 % 2 * 8 + t / 16 * 4 + t % 2 * 2 + t / 8 % 2; }

// One vector of a token spread over a warp (lane l: channels l EPL ..): codes of its pairs of channels and its block's scale byte.
template <int EPL>
SA_D uint32_t fp4_encode_vec(const uint32_t (&bits)[EPL], uint8_t (&codes)[EPL / 2]) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < EPL; ++i) top = max(top, bits[i] & 0x7fffu);
#pragma unroll
    for (int o = 1; o < 16 / EPL; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    const uint32_t b = fp4_scale_byte(top);
    const float s = fp4_scale(b), inv = fp4_inverse(s);
    uint32_t x[4] = {};
#pragma unroll
    for (int i = 0; i < EPL / 2; ++i) x[i] = bits[2 * i] | bits[2 * i + 1] << 16;
    const uint32_t w = fp4_codes(x, s, inv);
#pragma unroll
    for (int i = 0; i < EPL / 2; ++i) codes[i] = (uint8_t)(w >> (8 * i));
    return b;
}
// Writes token t (0 .. 31) into the half block at `half` (the keys' codes at its start, the values' at v_off).  A byte of value codes
// belongs to two tokens: the other one's nibble stays.
template <int D>
SA_D void write_token_fp4(uint8_t* half, size_t v_off, bool hadamard, int t, int lane, const uint16_t* krow, const uint16_t* vrow) {
    constexpr int EPL = D / 32;
    uint32_t kb[EPL], vb[EPL];
    load_vec_bits<EPL>(krow, lane, kb);
    load_vec_bits<EPL>(vrow, lane, vb);
    if (hadamard) {
        float x[EPL];
#pragma unroll
        for (int i = 0; i < EPL; ++i) x[i] = half_bits_to_float(kb[i]);
        hadamard_warp<EPL>(x, kb, lane);
    }
    const int m = lane * EPL;                       // first channel of this lane
    uint8_t codes[EPL / 2];
    uint32_t scale = fp4_encode_vec<EPL>(kb, codes);
    store_bytes<EPL / 2>(half + fp4_key_byte(t, m), codes);
    if (m % 16 == 0) half[fp4_key_scale(D, t, m)] = (uint8_t)scale;
    scale = fp4_encode_vec<EPL>(vb, codes);
    uint8_t* v = half + v_off;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
        uint8_t* at = v + fp4_value_byte(t, m + i);
        const uint32_t mine = (codes[i / 2] >> (4 * (i & 1))) & 0xfu, other = *at;
        *at = (uint8_t)((t & 1) ? (other & 0x0fu) | mine << 4 : (other & 0xf0u) | mine);
    }
    if (m % 16 == 0) v[fp4_value_scale(D, t, m)] = (uint8_t)scale;
}

// Half a page at once, keys or values of one head, by a warp.  A lane has a block of 16 channels, LPV lanes a vector, and the
// tokens t8, t8 + 8, t8 + 16, t8 + 24: whole rows are loaded and stored without shared memory, a lane's four key scales are one word of the page.
template <int D>
struct Fp4Half {
    static constexpr int LPV = D / 16, TPW = 32 / LPV, PARTS = 8 / TPW;      // lanes of a vector, tokens at a time, times to come to all of 8
    int blk, t8, lane;
    SA_D Fp4Half(int lane_, int part) : blk(lane_ % LPV), t8(part * TPW + lane_ / LPV), lane(lane_) {}
    SA_D uint8_t* key_words(uint8_t* half, int t) const { return half + (2 * (blk / 4)) * 512 + t * 16 + blk % 4 * 4; }     // + 512: the other 8 channels
    SA_D uint8_t* key_scales(uint8_t* half) const { return half + fp4_key_scale(D, t8, 16 * blk); }                          // of tokens t8 + 8 k
    SA_D uint8_t* value_words(uint8_t* v, int g) const { return v + blk / 2 * 512 + (4 * (t8 & 1) + g) * 64 + (t8 >> 1) * 16 + blk % 2 * 8; }
    SA_D uint8_t* value_scales(uint8_t* v) const { return v + 16 * D + blk / 2 * 64 + (t8 >> 1) * 16 + blk % 2 * 8; }

    // Walsh-Hadamard rotation of the vectors as hadamard_warp has it (the same sums in the same order), binary16 in and out; pairs of channels packed.
    SA_D void rotate(uint32_t (&h)[8]) const {
        f32x2 x[8];
        const f32x2 minus = pack_f32x2(-1.0f, -1.0f);
#pragma unroll
        for (int i = 0; i < 8; ++i) {                                        // channels 1 apart
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
            x[i] = pack_f32x2(__fadd_rn(f.x, f.y), __fsub_rn(f.x, f.y));
        }
#pragma unroll
        for (int st = 1; st < 8; st <<= 1)                                   // 2, 4, 8 apart
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if ((i & st) == 0) {
                    const f32x2 a = x[i], b = x[i + st];
                    x[i] = add2(a, b);
                    x[i + st] = ffma2(b, minus, a);                          // (a - b with the one rounding of a difference)
                }
#pragma unroll
        for (int st = 1; st < LPV; st <<= 1) {                               // other lanes
            const float sign = (lane & st) ? -1.0f : 1.0f;
            const f32x2 s2 = pack_f32x2(sign, sign);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float lo, hi;
                unpack_f32x2(x[i], &lo, &hi);
                x[i] = ffma2(x[i], s2, pack_f32x2(__shfl_xor_sync(0xffffffffu, lo, st), __shfl_xor_sync(0xffffffffu, hi, st)));
            }
        }
        const float scale = (D == 64) ? 0.125f : 0.088388346f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float lo, hi;
            unpack_f32x2(mul2(x[i], pack_f32x2(scale, scale)), &lo, &hi);
            const __half2 v = __floats2half2_rn(lo, hi);
            h[i] = *reinterpret_cast<const uint32_t*>(&v);
        }
    }
    // Codes of the lane's values w[k][channel / 8 % 2] (8 channels c % 8 in a word) -> bytes of pairs of tokens, out[g][t / 16] for the channels c % 8 =
    // 4 (t8 & 1) + g: the lanes of tokens t and t + 1 exchange halves of their words.
    SA_D void pair_tokens(const uint32_t (&w)[4][2], uint32_t (&out)[4][2]) const {
        const bool odd_token = t8 & 1;
        uint32_t lo[4], hi[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t mine = __byte_perm(w[k][0], w[k][1], odd_token ? 0x7632u : 0x5410u);
            const uint32_t other = __shfl_xor_sync(0xffffffffu, __byte_perm(w[k][0], w[k][1], odd_token ? 0x5410u : 0x7632u), LPV);
            const uint32_t even = odd_token ? other : mine, odd = odd_token ? mine : other;
            lo[k] = (even & 0x0f0f0f0fu) | ((odd << 4) & 0xf0f0f0f0u);       // channels g = 0, 2 of either half of the block
            hi[k] = ((even >> 4) & 0x0f0f0f0fu) | (odd & 0xf0f0f0f0u);       // g = 1, 3
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            out[0][k] = __byte_perm(lo[2 * k], lo[2 * k + 1], 0x6420);
            out[2][k] = __byte_perm(lo[2 * k], lo[2 * k + 1], 0x7531);
            out[1][k] = __byte_perm(hi[2 * k], hi[2 * k + 1], 0x6420);
            out[3][k] = __byte_perm(hi[2 * k], hi[2 * k + 1], 0x7531);
        }
    }
    SA_D void part_tokens(const uint32_t (&in)[4][2], uint32_t (&w)[4][2]) const {         // the way back
        const bool odd_token = t8 & 1;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t sel = k % 2 ? 0x7362u : 0x5140u;
            const uint32_t lo = __byte_perm(in[0][k / 2], in[2][k / 2], sel), hi = __byte_perm(in[1][k / 2], in[3][k / 2], sel);
            const uint32_t even = (lo & 0x0f0f0f0fu) | ((hi << 4) & 0xf0f0f0f0u), odd = ((lo >> 4) & 0x0f0f0f0fu) | (hi & 0xf0f0f0f0u);
            const uint32_t mine = odd_token ? odd : even, other = __shfl_xor_sync(0xffffffffu, odd_token ? even : odd, LPV);
            const uint32_t low = odd_token ? other : mine, high = odd_token ? mine : other;
            w[k][0] = __byte_perm(low, high, 0x5410);
            w[k][1] = __byte_perm(low, high, 0x7632);
        }
    }
    // Which nibbles of out[.][k] are tokens below n, which bytes of the scale words.
    SA_D uint32_t value_mask(int k, int n) const {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {                                        // (k: t / 16; i: t / 8 % 2 and t % 2)
            const int t = 16 * k + 8 * (i >> 1) + (t8 & ~1) + (i & 1);
            if (t < n) m |= (i & 1 ? 0xf0f0u : 0x0f0fu) << (16 * (i >> 1));
        }
        return m;
    }
    // The bits of x that `mask` has, by atomics where it has not all: sequences of one call that share a prefix share its pages, and where one ends
    // within a half that another fills on, both write the shared tokens (with the same bits), and the other's must not get lost between a
    // load and a store of this word.
    SA_D static void store_masked(uint8_t* at, uint32_t x, uint32_t mask) {
        uint32_t* p = reinterpret_cast<uint32_t*>(at);
        if (mask == 0xffffffffu) *p = x;
        else if (mask) {
            atomicAnd(p, ~mask);
            atomicOr(p, x & mask);
        }
    }
};
// Part `part` of the tile's first n tokens of K or V (rows of `pitch` elements) into the half page at `half`, whose value codes start at v_off.  What
// belongs to other tokens stays as it is; the parts share no word.  Keys in a rolled loop, the next token's block under way: unrolled, the code did not fit the instruction
// caches (20 001 tokens, 8 heads of 128, rotated: 46.7 -> 31.9 us, keys and values; the fill alone, in a graph, now 28.2).
template <int D, bool HAD>
SA_D void fp4_fill(uint8_t* half, size_t v_off, bool values, int part, const uint16_t* rows, size_t pitch, int n, int lane) {
    using F = Fp4Half<D>;
    const F f(lane, part);
    const bool wide = (reinterpret_cast<uintptr_t>(rows) & 31) == 0;
    auto load = [&](uint32_t (&x)[8], int t, int blk) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = 0u;
        if (t < n) load_32_bytes(rows + (size_t)t * pitch + 16 * blk, wide, x);
    };
    if (!values) {
        uint32_t next[2][8];
        load(next[0], f.t8, f.blk);
        load(next[1], f.t8 + 8, f.blk);
        uint32_t scales = 0, mask = 0;
#pragma unroll(HAD ? 1 : 4)
        for (int k = 0; k < 4; ++k) {
            uint32_t x[8], w[2];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = next[0][e];
                next[0][e] = next[1][e];
            }
            if (k < 2) load(next[1], f.t8 + 8 * (k + 2), f.blk);
            if constexpr (HAD) f.rotate(x);
            scales |= fp4_block(x, w) << (8 * k);
            if (8 * k + f.t8 < n) {
                uint8_t* at = f.key_words(half, 8 * k + f.t8);
                *reinterpret_cast<uint32_t*>(at) = w[0];
                *reinterpret_cast<uint32_t*>(at + 512) = w[1];
                mask |= 0xffu << (8 * k);
            }
        }
        F::store_masked(f.key_scales(half), scales, mask);
        return;
    }
    uint32_t in[4][8], w[4][2], scale[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) load(in[k], f.t8 + 8 * k, f.blk);
#pragma unroll
    for (int k = 0; k < 4; ++k) scale[k] = fp4_block(in[k], w[k]);
    uint8_t* v = half + v_off;
    uint32_t out[4][2];
    f.pair_tokens(w, out);
    if (n == kTileTokens) {
#pragma unroll
        for (int g = 0; g < 4; ++g) *reinterpret_cast<uint2*>(f.value_words(v, g)) = make_uint2(out[g][0], out[g][1]);
    } else {
        const uint32_t m0 = f.value_mask(0, n), m1 = f.value_mask(1, n);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            F::store_masked(f.value_words(v, g), out[g][0], m0);
            F::store_masked(f.value_words(v, g) + 4, out[g][1], m1);
        }
    }
    // scales: [t / 16][t % 2][t / 8 % 2]; the even token's lane stores those of the first 16 tokens, the odd one's the others
    const bool odd = f.t8 & 1;
    const uint32_t s0 = scale[0] | scale[1] << 8, s1 = scale[2] | scale[3] << 8;
    const uint32_t other = __shfl_xor_sync(0xffffffffu, odd ? s0 : s1, F::LPV);
    uint32_t mask = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)                                              // byte i: t % 2 = i / 2, t / 8 % 2 = i % 2
        if (16 * odd + 8 * (i & 1) + (f.t8 & ~1) + (i >> 1) < n) mask |= 0xffu << (8 * i);
    F::store_masked(f.value_scales(v) + 4 * odd, odd ? other | s1 << 16 : s0 | other << 16, mask);
}
// The way back: tokens first .. end - 1 of the half page to their rows (rows: that of token 0, from which only these are touched).
template <int D, bool HAD>
SA_D void fp4_read(const uint8_t* half_, size_t v_off, bool values, uint16_t* rows, int64_t pitch, int first, int end, int lane) {
    using F = Fp4Half<D>;
    uint8_t* half = const_cast<uint8_t*>(half_);
    const bool wide = (reinterpret_cast<uintptr_t>(rows) & 31) == 0;
    auto write = [&](const F& f, int k, uint32_t c0, uint32_t c1, uint32_t b, bool rotated) {
        const uint32_t s = b << 7 | b << 23;
        uint32_t x[8], lo[4], hi[4];
        fp4_to_half2(c0, lo);
        fp4_to_half2(c1, hi);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = mul_half2(lo[i], s);
            x[4 + i] = mul_half2(hi[i], s);
        }
        if (rotated) f.rotate(x);
        const int t = 8 * k + f.t8;
        if (t >= first && t < end) store_32_bytes(rows + t * pitch + 16 * f.blk, wide, x);
    };
    if (!values) {
        uint32_t w[F::PARTS * 4][2], scales[F::PARTS];
#pragma unroll
        for (int i = 0; i < 4 * F::PARTS; ++i) {
            const F f(lane, i >> 2);
            w[i][0] = *reinterpret_cast<const uint32_t*>(f.key_words(half, 8 * (i & 3) + f.t8));
            w[i][1] = *reinterpret_cast<const uint32_t*>(f.key_words(half, 8 * (i & 3) + f.t8) + 512);
        }
#pragma unroll
        for (int part = 0; part < F::PARTS; ++part) scales[part] = *reinterpret_cast<const uint32_t*>(F(lane, part).key_scales(half));
        if constexpr (HAD) {                                                 // rolled: the rotation is long
#pragma unroll 1
            for (int i = 0; i < 4 * F::PARTS; ++i) {
                write(F(lane, i >> 2), i & 3, w[0][0], w[0][1], scales[0] >> (8 * (i & 3)) & 0xffu, true);
#pragma unroll
                for (int k = 0; k + 1 < 4 * F::PARTS; ++k) {
                    w[k][0] = w[k + 1][0];
                    w[k][1] = w[k + 1][1];
                }
                if ((i & 3) == 3) scales[0] = scales[F::PARTS - 1];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4 * F::PARTS; ++i) write(F(lane, i >> 2), i & 3, w[i][0], w[i][1], scales[i >> 2] >> (8 * (i & 3)) & 0xffu, false);
        }
        return;
    }
    uint32_t w[F::PARTS][4][2], scales[F::PARTS][2];
#pragma unroll
    for (int part = 0; part < F::PARTS; ++part) {
        const F f(lane, part);
#pragma unroll
        for (int k = 0; k < 2; ++k) scales[part][k] = *reinterpret_cast<const uint16_t*>(f.value_scales(half + v_off) + 4 * k + 2 * (f.t8 & 1));
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const uint2 x = *reinterpret_cast<const uint2*>(f.value_words(half + v_off, g));
            w[part][g][0] = x.x;
            w[part][g][1] = x.y;
        }
    }
#pragma unroll
    for (int part = 0; part < F::PARTS; ++part) {
        const F f(lane, part);
        uint32_t c[4][2];
        f.part_tokens(w[part], c);
#pragma unroll
        for (int k = 0; k < 4; ++k) write(f, k, c[k][0], c[k][1], scales[part][k / 2] >> (8 * (k & 1)) & 0xffu, false);
    }
}

}  // namespace sa
