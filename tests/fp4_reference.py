"""The 4-bit cache in numpy, from its definition in the C header and 64-bit arithmetic: codes, their places in a page, attention."""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def round_to_even_multiple(x, step):
    return np.rint(x / step) * step


def scale_bytes(x):
    """x [..., 16] -> the block's scale byte."""
    t = np.abs(x.astype(np.float64)).max(-1) / 6.0
    exponent = np.floor(np.log2(np.maximum(t, 2.0 ** -14)))
    s = np.minimum(round_to_even_multiple(t, 2.0 ** (exponent - 3)), 10240.0)
    bits = s.astype(np.float16).view(np.uint16)
    assert np.all(bits.view(np.float16).astype(np.float64) == s) and np.all(bits % 128 == 0)
    return (bits >> 7).astype(np.uint8)


def scales(b):
    return (b.astype(np.uint16) << 7).view(np.float16).astype(np.float64)


def encode(x):
    """x [..., d] binary16 -> codes [..., d], scale bytes [..., d / 16].  A zero's sign bit is left out."""
    blocks = x.astype(np.float64).reshape(*x.shape[:-1], -1, 16)
    b = scale_bytes(blocks)
    s = scales(b)[..., None]
    r = np.abs(blocks) / np.where(s > 0, s, 1.0) * (s > 0)
    gap = np.abs(r[..., None] - LEVELS)
    even_first = gap + np.where(np.arange(8) % 2, 1e-9, 0.0)          # of two equally near levels the even code (others are > 1e-6 apart)
    code = np.argmin(even_first, -1)
    code = code + 8 * ((blocks < 0) & (code > 0))
    return code.astype(np.uint8).reshape(x.shape), b


def decode(code, b):
    v = LEVELS[code & 7] * np.where(code & 8, -1.0, 1.0)
    return (v.reshape(*v.shape[:-1], -1, 16) * scales(b)[..., None]).reshape(v.shape)


def quantised(x):
    """The numbers that binary16 vectors are held as (float64)."""
    return decode(*encode(x))


def places(d):
    """Byte and nibble of every (token, channel) in half a page: key codes, key scales, value codes, value scales (arrays [32, d])."""
    t, c = np.meshgrid(np.arange(32), np.arange(d), indexing="ij")
    key = (2 * (c // 64) + c // 8 % 2) * 512 + t * 16 + c // 16 % 4 * 4 + c % 8 // 2
    key_scale = 16 * d + c // 64 * 128 + c // 16 % 4 * 32 + t % 8 * 4 + t // 8
    v0 = 18 * d
    value = v0 + c // 32 * 512 + c % 8 * 64 + t % 8 // 2 * 16 + c // 16 % 2 * 8 + t // 16 * 4 + t // 8 % 2 * 2 + c // 8 % 2
    value_scale = v0 + 16 * d + c // 32 * 64 + t % 8 // 2 * 16 + c // 16 % 2 * 8 + t // 16 * 4 + t % 2 * 2 + t // 8 % 2
    return (key, c % 2), key_scale, (value, t % 2), value_scale


def unpack(half, d):
    """Half a page (36 d bytes) -> codes and scale bytes of keys and values, [32, d] and [32, d / 16]."""
    (k, kn), ks, (v, vn), vs = places(d)
    return (half[k] >> (4 * kn)) & 15, half[ks][:, ::16], (half[v] >> (4 * vn)) & 15, half[vs][:, ::16]


def hadamard(x):
    """The rotation of the definition: 32-bit butterflies of channels 1, 2, 4, ... apart, rounded to binary16."""
    x = x.astype(np.float32)
    d = x.shape[-1]
    i = np.arange(d)
    h = 1
    while h < d:
        x = np.where(i & h, x[..., i ^ h] - x, x + x[..., i ^ h]).astype(np.float32)
        h *= 2
    return (x * np.float32(0.125 if d == 64 else 0.088388346)).astype(np.float16)


def attention(Q, K, V, cu, groups):
    """softmax(Q K^T / sqrt(d)) V in 64 bits; Q [B, Hq, d], K, V [n, Hkv, d]; and what errors are measured against: the sums of
    |q k| / sqrt(d) of the hardest key [B, Hq, 1], of p |v| and of |v| times the largest p [B, Hq, d]."""
    B, Hq, d = Q.shape
    O, hard, size, flat = np.zeros((B, Hq, d)), np.zeros((B, Hq, 1)), np.zeros((B, Hq, d)), np.zeros((B, Hq, d))
    for b in range(B):
        k, v = K[cu[b]:cu[b + 1]].astype(np.float64), V[cu[b]:cu[b + 1]].astype(np.float64)
        if not len(k):
            continue
        for h in range(Hq):
            q, kh, vh = Q[b, h].astype(np.float64), k[:, h // groups], v[:, h // groups]
            z = kh @ q / np.sqrt(d)
            p = np.exp(z - z.max())
            p /= p.sum()
            O[b, h], size[b, h], hard[b, h] = p @ vh, p @ np.abs(vh), (np.abs(kh) @ np.abs(q)).max() / np.sqrt(d)
            flat[b, h] = np.abs(vh).sum(0) * p.max()
    return O, (hard, size, flat)


def tolerance(against, d, longest):
    """Of the attention's FP32 sums.  A logit is a sum of d products, each step cut off or rounded by at most 2^-23 of the sum of magnitudes, and
    is scaled with three more roundings: it is off by (d + 3) 2^-23 `hard`, which moves a weight, and the mean, by twice that, relatively;
    a weight itself (exponent's argument of at most 28 bits before the point apart, 2^-22 of ex2, two binary16 terms: 2^-21); sums of `longest` keys in
    chains of 16 products a step, two steps for two terms, cut off by 2^-23 each.
    A weight far below the largest is off by an absolute 2^-38 of that one: the largest, scaled by 2^14, lies at 2^13 at least (the reference is
    the largest logit so far, rounded up), and the second binary16 term is rounded to half a step of the subnormal numbers, 2^-25."""
    hard, size, flat = against
    return (2 * (d + 3) * 2.0 ** -23 * hard + 2.0 ** -19 + longest / 8 * 2.0 ** -23) * size + 2.0 ** -38 * flat + 1e-30
