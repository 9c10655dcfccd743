"""The attention of the 4-bit cache in numpy with the kernels' roundings: logits and outputs as chains of products over 16 channels or keys whose
sums are cut off to 24 bits, weights in FP32, entering the second product as the sum of two binary16 terms, the products of a tile of keys summed
from zero and added to those before by an FP32 addition.  And, from the same formulas, how far such outputs are off in the mean square."""
import numpy as np


def cut(x):
    """float64 -> float32 towards zero."""
    y = x.astype(np.float32)
    return np.where(np.abs(y.astype(np.float64)) > np.abs(x), np.nextafter(y, np.float32(0)), y).astype(np.float32)


def logits(q, k):
    """q [G, d], k [T, d] (numbers of binary16) -> [G, T] float32, and the sum of |partial sum| over the steps, [G, T] float64."""
    q, k = q.astype(np.float64), k.astype(np.float64)
    s, reach = np.zeros((len(q), len(k)), np.float32), 0.0
    for c in range(0, q.shape[1], 16):
        x = s.astype(np.float64) + q[:, c:c + 16] @ k[:, c:c + 16].T
        s, reach = cut(x), reach + np.abs(x)
    return s, reach


def attention(q, k, v, *, tile, chains, terms=2, fine=True):
    """Outputs [G, d] of one query group; `chains` warps share the tiles.  terms=1: without the second binary16 term of a weight; fine=False: products
    are added to those of the tiles before within the matrix unit."""
    G, d = q.shape
    T = len(k)
    s, _ = logits(q, k)
    qs = np.float32(np.log2(np.e) / np.sqrt(d))
    R = np.ceil((s * qs).max(1, keepdims=True))
    x = (s.astype(np.float64) * np.float64(qs) - (R - 14)).astype(np.float32)
    w = np.exp2(x.astype(np.float64)).astype(np.float32)
    n = -(-T // (tile * chains)) * tile * chains
    w = np.pad(w, ((0, 0), (0, n - T))).reshape(G, -1, chains, tile).astype(np.float32)
    vv = np.pad(v.astype(np.float64), ((0, n - T), (0, 0))).reshape(-1, chains, tile, d)
    hi = w.astype(np.float16)
    lo = (w - hi.astype(np.float32)).astype(np.float16)
    acc, l = np.zeros((chains, G, d), np.float32), np.zeros((chains, G), np.float32)
    for t in range(w.shape[1]):
        own = np.zeros_like(acc) if fine else acc
        for j in range(0, tile, 16):
            for term in (hi, lo)[:terms]:
                own = cut(own + np.einsum("gck,ckd->cgd", term[:, t, :, j:j + 16].astype(np.float64), vv[t, :, j:j + 16]))
        acc = acc + own if fine else own
        for j in range(0, tile, 8):                               # (a lane has a few of the tile's keys; their sums are added at the end)
            l = l + w[:, t, :, j:j + 8].sum(-1, dtype=np.float32).T
    return acc.astype(np.float64).sum(0) / l.astype(np.float64).sum(0)[:, None]


def exact(q, k, v):
    z = q.astype(np.float64) @ k.astype(np.float64).T / np.sqrt(q.shape[1])
    p = np.exp(z - z.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    return p, p @ v.astype(np.float64)


def mean_square_bound(q, k, tile, tiles):
    """How far outputs may be off, root mean square relative to theirs, where values are independent of the weights and have mean zero.

    With such values sum_i p_i e_i v_i has the mean square sum_i p_i^2 e_i^2 of sum_i p_i v_i's sum_i p_i^2, whatever the errors e_i of the weights are: no matter how
    they depend on one another, and independent of the number of keys.  e_i: the logit, cut off by 2^-23 of the sum so far in every step; the exponent's
    argument, rounded by 2^-24 of its size; ex2, 2^-22; the two terms, 2^-23.  All at their largest, so the bound is not a guess of how they fall.
    The sums: `tile` / 16 steps for two terms, each cut off by 2^-23 of a sum that grows to the tile's as the root of its steps (2/3 of them on the
    whole); an addition of 2^-24 for every tile of a chain, of which only the sums' mean square counts as they are rounded to nearest:
    sqrt(tiles / 2) 2^-24, as those too grow as the root; and the same for the normaliser, a chain of tile / 8 additions a tile."""
    d = q.shape[1]
    s, reach = logits(q, k)
    z = s.astype(np.float64) / np.sqrt(d)
    p = np.exp(z - z.max(1, keepdims=True))
    x = (z - z.max(1, keepdims=True)) * np.log2(np.e) + 15
    e = 2.0 ** -23 * reach / np.sqrt(d) + np.log(2) * 2.0 ** -24 * np.abs(x) + 2.0 ** -22 + 2.0 ** -23
    weights = np.sqrt((p * p * e * e).sum(1) / (p * p).sum(1))
    sums = 2 * tile / 16 * 2 / 3 * 2.0 ** -23 + np.sqrt(tiles / 2) * 2.0 ** -24 + np.sqrt(tiles * tile / 8 / 2) * 2.0 ** -24
    return np.sqrt((weights ** 2).mean()) + sums
