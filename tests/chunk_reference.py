"""Attention of chunks of new tokens in 64 bits, from the numbers that a cache holds, and how far a result may be from it."""
import numpy as np
import torch

import fp4_reference as fp4
from paper_2609_09208_b200 import binding as sa


def queries(cfg, Q):
    """What stands for the queries [n, heads, d] (binary16, numpy) of a chunk: rotated and rounded to 8 bits where the code says so."""
    if cfg.flags & 1:
        Q = fp4.hadamard(Q)
    if cfg.code in (sa.SA_KV_FP16, sa.SA_KV_FP4):
        return Q.astype(np.float64)
    x = Q.astype(np.float32)
    top = np.abs(x).max(-1, keepdims=True)
    inv = np.divide(np.float32(127), top, out=np.zeros_like(top), where=top > 0)
    return np.clip(np.rint(x * inv), -127, 127).astype(np.float64) * top.astype(np.float64) / 127


def attend(cfg, Q, K, V, before, window=0, sinks=0, there=None, out_step=2.0 ** -11):
    """One sequence: queries [n, Hq, d] (numbers) at places before, before + 1, ..; keys and values [T, Hkv, d] of its tokens 0 .. T - 1, of which `there` (bool [T]) says which
    there are.  Returns O [n, Hq, d] and the error that it may have, both 64 bits.

    The error: a weight is rounded to binary16 (2^-11 of it, or 2^-25 of numbers of which the row's largest is at least 2^7), and so may be the sum that they are divided by.  Its
    exponent is off by the sum's error, d + 8 roundings of 2^-23 (the matrix unit cuts off) of the sum of magnitudes, and by 2^-22 for the power itself.  The output is rounded once."""
    n, Hq, d = Q.shape
    T, Hkv, _ = K.shape
    if T == 0 or n == 0:
        return np.zeros((n, Hq, d)), np.zeros((n, Hq, d))
    cuda = lambda x: torch.as_tensor(x, dtype=torch.float64, device="cuda")
    i, j = before + torch.arange(n, device="cuda")[:, None], torch.arange(T, device="cuda")[None]
    seen = j <= i
    if window:
        seen &= (j > i - window) | (j < sinks)
    if there is not None:
        seen &= torch.as_tensor(there, device="cuda")[None]
    O, off = np.zeros((n, Hq, d)), np.zeros((n, Hq, d))
    for h in range(Hq):
        q, k, v = cuda(Q[:, h]), cuda(K[:, h * Hkv // Hq]), cuda(V[:, h * Hkv // Hq])
        z = (q @ k.T / d ** 0.5).masked_fill(~seen, -torch.inf)
        reach = ((q.abs() @ k.abs().T) / d ** 0.5).masked_fill(~seen, 0.0).amax(-1, keepdim=True)
        w = torch.exp(z - z.amax(-1, keepdim=True).clamp(min=-1e300))
        w = torch.where(seen, w, 0.0) / w.masked_fill(~seen, 0.0).sum(-1, keepdim=True).clamp(min=1e-300)
        o, size = w @ v, w @ v.abs()
        eps = 2.0 ** -11 + (d + 8) * 2.0 ** -23 * reach + 2.0 ** -22
        tail = T * 2.0 ** -32 * v.abs().amax()
        O[:, h] = o.cpu().numpy()
        off[:, h] = (1.02 * (eps * (size + o.abs()) + tail) + (out_step * o.abs()).clamp(min=2.0 ** -25)).cpu().numpy()
    return O, off
