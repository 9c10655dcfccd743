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

// x / s, correctly rounded where it matters (see above): exact for quotients of a few bits, within an ulp otherwise.
SA_HD float fp4_quotient(float x, float s, float inv) {
    const float r = x * inv;
#ifdef __CUDA_ARCH__
    return __fmaf_rn(__fmaf_rn(-r, s, x), inv, r);
#else
    return fmaf(fmaf(-r, s, x), inv, r);
#endif
}
// Scale byte of a block whose largest magnitude has the binary16 bits `amax`.
SA_D uint32_t fp4_scale_byte(uint32_t amax) {
    const float t = fp4_quotient(half_bits_to_float(amax), 6.0f, 1.0f / 6.0f);
    const uint32_t u = __float_as_uint(t);
    const uint32_t normal = ((u + 0x7ffffu + ((u >> 20) & 1u)) >> 20) - (112u << 3);
    const uint32_t b = t >= 0x1p-14f ? normal : (uint32_t)__float2int_rn(t * 0x1p17f);
    return min(b, kFp4ScaleMost);
}
SA_D float fp4_scale(uint32_t byte) { return half_bits_to_float(byte << 7); }
// Codes of 8 channels (pairs of binary16), the first in the lowest nibble.
SA_D uint32_t fp4_codes(const uint32_t (&x)[4], float s, float inv) {
    float q[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        q[2 * i] = fp4_quotient(half_bits_to_float(x[i] & 0xffffu), s, inv);
        q[2 * i + 1] = fp4_quotient(half_bits_to_float(x[i] >> 16), s, inv);
    }
    uint32_t w;
    asm("{.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\tmov.b32 %0, {a, b, c, d};}"
        : "=r"(w)
        : "f"(q[0]), "f"(q[1]), "f"(q[2]), "f"(q[3]), "f"(q[4]), "f"(q[5]), "f"(q[6]), "f"(q[7]));
    return w;
}
// A block of 16 channels (pairs of binary16): codes of the first 8, and of the others to `second`; its scale byte to `scale` (unless null).
SA_D uint32_t fp4_block(const uint32_t (&x)[8], uint32_t* second, uint8_t* scale) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = __vmaxu2(top, x[i] & 0x7fff7fffu);       // two magnitudes at a time; they order like their bits
    const uint32_t b = fp4_scale_byte(max(top & 0xffffu, top >> 16));
    const float s = fp4_scale(b), inv = s > 0.0f ? __frcp_rn(s) : 0.0f;
    if (scale) *scale = (uint8_t)b;
    const uint32_t lo[4] = {x[0], x[1], x[2], x[3]}, hi[4] = {x[4], x[5], x[6], x[7]};
    *second = fp4_codes(hi, s, inv);
    return fp4_codes(lo, s, inv);
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
    const float s = fp4_scale(b), inv = s > 0.0f ? __frcp_rn(s) : 0.0f;
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

// The 8 x 8 nibbles that the lanes t, t ^ 1, t ^ 8, t ^ 16, ... hold in a word each, transposed: nibble i of the lane whose bits
// 0, 3, 4 are the bits of j goes to nibble j of the lane of i.
SA_D uint32_t fp4_transpose(uint32_t w, int lane) {
    uint32_t p = __shfl_xor_sync(0xffffffffu, w, 1);
    w = (lane & 1) ? (w & 0xf0f0f0f0u) | ((p >> 4) & 0x0f0f0f0fu) : (w & 0x0f0f0f0fu) | ((p << 4) & 0xf0f0f0f0u);
    p = __shfl_xor_sync(0xffffffffu, w, 8);
    w = __byte_perm(w, p, (lane & 8) ? 0x3715u : 0x6240u);
    p = __shfl_xor_sync(0xffffffffu, w, 16);
    return __byte_perm(w, p, (lane & 16) ? 0x3276u : 0x5410u);
}
// The lane's number among the eight that share a piece of 16 bytes of value codes: also the channel (mod 8) whose piece it moves.
SA_D int fp4_piece_of(int lane) { return (lane & 1) | (lane >> 2 & 2) | (lane >> 2 & 4); }

}  // namespace sa
