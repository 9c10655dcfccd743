"""Timed cases of what a serving loop does with several new tokens of a sequence at a time: from a layer's projections into the cache
(``append_qkv``), attention of the new tokens over the paged cache (``chunk_attention``), and the same with a sliding window and a few first
tokens that stay visible.

Kinds of case:

  append   norms of queries and keys for each head, rotation by the token's position, queries out, keys and values into the cache behind what it
           holds, for a chunk of new tokens per sequence; and the new tokens as the cache holds them (``read_kv``)
  chunk    attention of the last tokens of every sequence over the cache, each token over what is not behind it
  window   the same, a token sees its last `window` tokens (itself among them) and the first `sinks` of the sequence

Shapes: 32 query / 4 KV heads of 64 channels, 32 / 8 heads of 128, and the odd ones between; chunks of one token to some thousands, caches of up to 32 768 tokens
in the codes that a cache can have.

The numbers that a cache holds:
  FP16    keys and values as they are
  POTM4   a key's scale is its largest magnitude s; a channel stands for s * +-(1 + j / 16) * 2^-e, the nearest such number in the logarithm, e = 0 .. 6, or 0
          where the grid continued to e = 7 is nearest;  POT4: the same without j
  INT8    a key channel is round(x * 127 / s) * s / 127
  FP4     a block of 16 channels has the scale max|x| / 6 rounded to 5 bits of exponent and 3 of mantissa, a channel is the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times it
  values of POT4, POTM4 and INT8: round(x * 2^g) * 2^-g with the largest g for which the largest magnitude stays within 127
and over POT4, POTM4 and INT8 a query is rounded to 127 steps of its largest magnitude first.

A page of one KV head holds 64 tokens as two halves of 32 (t: token in it): FP16, keys then values, in chunks of 8 channels, [d / 8][32 tokens][8]; POTM4 and INT8 the codes
in chunks of 16 bytes, [d / 16][32][16], POT4 of 32 nibbles, [d / 32][32][16], then 4 bytes a token (binary16 s, g, 0), then the values as INT8 [d / 16][32][16]; FP4:
  key codes     [d / 32 chunks][32 tokens][16 bytes]: word i of chunk c holds channels 64 (c / 2) + 16 i + 8 (c % 2) .. + 7, two a byte
  key scales    [d / 64][block % 4][token % 8][token / 8]
  value codes   [d / 32][channel % 8][token % 8 / 2][channel / 16 % 2][token / 16][token / 8 % 2][channel / 8 % 2], a byte: tokens 2 i, 2 i + 1
  value scales  [d / 32][token % 8 / 2][channel / 16 % 2][token / 16][token % 2][token / 8 % 2]
"""
import math

import numpy as np
import torch

own = False                              # set by who times: False: elementary torch operations, True: the library's kernels

POT4, POTM4, INT8, FP16, FP4 = 0, 4, 8, 16, 32      # codes of a cache
F16, BF16, F32 = 0, 1, 2                            # types of a projection's output, and of the attention's (F16, BF16)
TYPES = (torch.float16, torch.bfloat16, torch.float32)
EQUAL, ONE, SPREAD = 0, 1, 2                        # chunks: all of `new` tokens; one of `new`, the others of 1; from 1 to `new`


def _case(kind, *, d=64, q_heads=32, kv_heads=4, batch=1, tokens=1024, shortest=0, new=1, mix=EQUAL, code=POTM4, hadamard=False, dtype=BF16, norm=True,
          neighbours=False, window=0, sinks=0, **more):
    """tokens: length of every sequence, its chunk included, or the longest of a ragged batch whose shortest is `shortest` (0: all equal).  new, mix: its chunks.
    dtype: of the projections (append), of the output (chunk, window)."""
    return dict(more, kind=kind, d=d, q_heads=q_heads, kv_heads=kv_heads, batch=batch, tokens=tokens, shortest=shortest, new=new, mix=mix, code=code,
                hadamard=hadamard, dtype=dtype, norm=norm, neighbours=neighbours, window=window, sinks=sinks)


def listed():
    return [
        # a decode step of one chat
        _case("append", tokens=1025, dtype=F16, norm=False, name="append_token"),
        # a decode step of a large batch, 4-bit cache
        _case("append", d=128, kv_heads=8, batch=32, tokens=4096, code=FP4, name="append_b32"),
        # the next chunk of a long prompt, at an odd place of its page
        _case("append", tokens=3049, new=2048, name="append_chunk_2k"),
        # prompts of several sequences, FP32 projections, rotated keys
        _case("append", d=128, kv_heads=8, batch=4, tokens=9001, shortest=6000, new=5001, mix=SPREAD, code=INT8, hadamard=True, dtype=F32, name="append_ragged_5001"),
        # five drafted tokens of one chat are checked: latency
        _case("chunk", tokens=4099, new=5, dtype=F16, name="chunk_draft_4k"),
        # drafts of a batch over long 4-bit caches
        _case("chunk", batch=16, tokens=16384, shortest=3001, new=8, code=FP4, name="chunk_drafts_b16"),
        # a prompt of a model with 128 channels a head, unquantised cache
        _case("chunk", d=128, kv_heads=8, tokens=4096, new=4096, code=FP16, name="chunk_prompt_4k"),
        # the last chunk of a long prompt: the largest
        _case("chunk", tokens=32768, new=2048, name="chunk_2k_32k"),
        # continuous batching: a chunk of one prompt beside the single tokens of others
        _case("chunk", batch=8, tokens=8192, shortest=1500, new=511, mix=ONE, code=INT8, name="chunk_mixed_b8"),
        # a token of one chat with a short window: the smallest call
        _case("window", q_heads=8, kv_heads=1, tokens=1000, window=256, sinks=1, dtype=F16, name="window_token"),
        # a decode step of a large batch of long sequences
        _case("window", batch=32, tokens=32768, window=4096, sinks=4, name="window_b32_32k"),
        # a chunk of a long prompt, the window shorter than the chunk
        _case("window", d=128, kv_heads=8, tokens=20001, new=4001, code=FP4, window=1024, sinks=4, name="window_chunk_4k"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["append", "append", "chunk", "chunk", "chunk", "window", "window"])
    d, q_heads, kv_heads = rng.choice([(64, 32, 4), (64, 32, 4), (128, 32, 8), (64, 8, 2), (64, 1, 1), (128, 16, 16), (128, 40, 8), (64, 12, 1)])
    code, mix = rng.choice([POT4, POTM4, POTM4, INT8, FP16, FP4]), rng.choice([EQUAL, EQUAL, ONE, SPREAD])
    batch, hadamard = rng.choice([1, 1, 1, 2, 3, 8, 13, 32]), code != FP16 and rng.random() < 0.3
    if kind == "append":
        new = _log_int(rng, 1, max(1, 2 ** 25 // (d * (q_heads + 2 * kv_heads) * batch))) if rng.random() < 0.7 else 1
        return _case(kind, d=d, q_heads=q_heads, kv_heads=kv_heads, batch=batch, tokens=new + rng.randint(0, 2000), new=new, mix=mix, code=code, hadamard=hadamard,
                     dtype=rng.choice([F16, BF16, F32]), norm=rng.random() < 0.6, neighbours=rng.random() < 0.4)
    tokens = _log_int(rng, 100, min(32768, 2 ** 29 // (batch * q_heads * d // 64)))
    # scores of the plain form (of padded chunks): at most a half of the largest listed case's
    new = min(tokens, _log_int(rng, 1, max(1, min(4096, 2 ** 30 // (batch * tokens * q_heads)) * 64 // d)) if rng.random() < 0.75 else 1)
    window = _log_int(rng, 16, 4096) if kind == "window" else 0
    return _case(kind, d=d, q_heads=q_heads, kv_heads=kv_heads, batch=batch, tokens=tokens, shortest=rng.choice([0, max(1, tokens // 5)]) if batch > 1 else 0, new=new, mix=mix,
                 code=code, hadamard=hadamard, dtype=rng.choice([F16, BF16]), window=window, sinks=rng.choice([0, 1, 4, 4, 100]) if window else 0)


def _lens(case):
    """Tokens and new tokens of every sequence.  Lengths: all equal, or spread evenly from the shortest to the longest in a mixed order."""
    B, T, lo, new = case["batch"], case["tokens"], case["shortest"], case["new"]
    order = (np.arange(B) * 7 + 3) % B if B % 7 else np.arange(B)[::-1]
    lens = np.linspace(lo, T, B).astype(np.int64)[order] if lo and B > 1 else np.full(B, T, dtype=np.int64)
    if case["mix"] == SPREAD and B > 1:
        n = np.linspace(1, new, B).astype(np.int64)[order]
    else:
        n = np.full(B, new if case["mix"] == EQUAL or B == 1 else 1, dtype=np.int64)
        n[int(lens.argmax())] = new
    return lens, np.minimum(n, lens)


# ---- inputs -------------------------------------------------------------------------------------------------------------------------

def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _half_bytes(case):
    d, code = case["d"], case["code"]
    return 32 * {FP16: 4 * d, FP4: d + d // 8, POT4: d // 2 + 4 + d}.get(code, 2 * d + 4)


def _key_bytes(case):
    return 32 * case["d"] // (2 if case["code"] == POT4 else 1)


def _pages(case, gen, n_pages):
    """A pool of full pages: [page, KV head, half, bytes], of random codes and of scales such as keys and values of a layer have."""
    H, d, code = case["kv_heads"], case["d"], case["code"]
    n = n_pages * H * 2
    if code == FP16:
        x = _normal(gen, n, 2, d // 8, 32, 8)
        x[:, 0] *= torch.exp(0.5 * _normal(gen, 1, d // 8, 1, 8))
        return x.half().view(torch.uint8).reshape(n_pages, H, 2, -1)
    half = torch.randint(0, 256, (n, _half_bytes(case)), generator=gen, device="cuda", dtype=torch.uint8)
    if code == FP4:                                            # scale bytes around 1 / 4: code * scale up to 1.5 or so
        for lo in (16 * d, 34 * d):
            half[:, lo:lo + 2 * d] = torch.randint(96, 112, (n, 2 * d), generator=gen, device="cuda").byte()
        return half.reshape(n_pages, H, 2, -1)
    k = _key_bytes(case)
    if code == POTM4:                                          # (an exponent field of 0 is the zero code, of which no other bit is set)
        half[:, :k].mul_((half[:, :k] & 7) > 0)
    if code == POT4:
        lo, hi = half[:, :k] & 15, half[:, :k] >> 4
        half[:, :k] = lo * ((lo & 7) > 0) + (hi * ((hi & 7) > 0) << 4)
    meta = half[:, k:k + 128].view(torch.int16)                                      # scale of the key, exponent of the value's scale
    meta[:, 0::2] = (1.0 + _normal(gen, n, 32).abs()).half().view(torch.int16)
    meta[:, 1::2] = torch.randint(4, 7, (n, 32), generator=gen, device="cuda").short()
    return half.reshape(n_pages, H, 2, -1)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    B, Hq, Hkv, d = case["batch"], case["q_heads"], case["kv_heads"], case["d"]
    lens, new = _lens(case)
    pages = (lens + 63) // 64
    table = np.full((B, int(pages.max())), -1, dtype=np.int32)
    table[np.arange(table.shape[1])[None] < pages[:, None]] = np.random.Generator(np.random.PCG64(seed)).permutation(int(pages.sum()))
    n = int(new.sum())
    s = dict(case=case, n=n, cu=np.concatenate([[0], np.cumsum(new)]), before=lens - new)
    s["table"] = torch.from_numpy(table).cuda()
    s["seq"] = torch.from_numpy(np.repeat(np.arange(B), new)).cuda()                 # of every new token: its sequence, place in the chunk and in the sequence
    s["at"] = torch.from_numpy(np.concatenate([np.arange(k) for k in new])).cuda()
    s["pos"] = torch.from_numpy(np.concatenate([np.arange(t - k, t) for t, k in zip(lens, new)]).astype(np.int32)).cuda()
    s["lens0"] = torch.from_numpy((lens - new if case["kind"] == "append" else lens).astype(np.int32)).cuda()
    s["lens"] = s["lens0"].clone()
    s["pages"] = _pages(case, gen, int(pages.sum()))
    if case["kind"] == "append":
        t = TYPES[case["dtype"]]
        s["x"] = _normal(gen, n, (Hq + 2 * Hkv) * d).to(t)                           # queries, keys and values of a token side by side
        s["inv_freq"] = (10000.0 ** (-torch.arange(d // 2, device="cuda", dtype=torch.float64) * 2 / d)).float()
        s["wq"], s["wk"] = ((1.0 + 0.2 * _normal(gen, d)).to(t) if case["norm"] else None for _ in "qk")
        s["Q"], s["K"], s["V"] = (torch.zeros(n, h, d, dtype=torch.float16, device="cuda") for h in (Hq, Hkv, Hkv))
    else:
        s["Q"] = _normal(gen, n, Hq, d).half()
        s["O"] = torch.zeros(n, Hq, d, dtype=TYPES[case["dtype"]], device="cuda")
    if own:
        _handles(s)
    torch.cuda.synchronize()
    return s


def _handles(s):
    """What a program keeps from call to call: the configuration, the cache's handle, the rotation's tables, the workspace."""
    from paper_2609_09208_b200 import binding as sa
    case = s["case"]
    d, Hq, Hkv = case["d"], case["q_heads"], case["kv_heads"]
    s["sa"], s["cfg"] = sa, sa.make_config(d, Hq, Hkv, case["code"], nibble=case["code"] == POT4, hadamard=case["hadamard"])
    s["handle"] = sa.make_cache(s["pages"], s["table"], s["lens"], len(s["pages"]))
    if case["kind"] == "append":
        s["rotary"] = sa.Rotary(s["cfg"], s["inv_freq"], dtype=TYPES[case["dtype"]], pairs="neighbours" if case["neighbours"] else "halves", norm=case["norm"],
                                eps=1e-6, q_weight=s["wq"], k_weight=s["wk"])
        s["qkv"] = [x.unflatten(1, (-1, d)) for x in s["x"].split([Hq * d, Hkv * d, Hkv * d], 1)]
    else:
        s["workspace"] = torch.empty(sa.chunk_workspace_bytes(s["cfg"], case["batch"], s["n"]), dtype=torch.uint8, device="cuda")


# ---- the operators ------------------------------------------------------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    sa, case = s["sa"], s["case"]
    if case["kind"] == "append":
        s["lens"].copy_(s["lens0"])                            # as a program does that drops rejected tokens
        sa.append_qkv(s["rotary"], s["handle"], *s["qkv"], s["pos"], s["cu"], s["Q"])
        sa.read_kv(s["cfg"], s["handle"], s["before"], s["cu"], s["K"], s["V"])
        return {"Q": s["Q"], "K": s["K"], "V": s["V"], "lens": s["lens"]}
    sa.chunk_attention(s["cfg"], s["handle"], s["Q"], s["O"], s["workspace"], s["cu"], window=case["window"], sinks=case["sinks"])
    return {"O": s["O"]}


def _rotate_hadamard(x):
    """Walsh-Hadamard rotation of the last axis, in 32 bits, in the order that the cache's definition fixes."""
    x, d = x.float(), x.shape[-1]
    for h in (1 << i for i in range(d.bit_length() - 1)):
        a, b = x.unflatten(-1, (-1, 2, h)).unbind(-2)
        x = torch.stack([a + b, a - b], -2).flatten(-3)
    return x * torch.tensor(1.0 / math.sqrt(d), dtype=torch.float32)


def _run_plain(s):
    return _append_plain(s) if s["case"]["kind"] == "append" else _attend_plain(s)


def _held_fp4(x):
    """Keys or values as the 4-bit cache holds them.  The decisions are exact in 32 bits."""
    x = x.float().unflatten(-1, (-1, 16))
    t = x.abs().amax(-1, keepdim=True) / 6.0
    step = torch.exp2(torch.floor(torch.log2(t.clamp(min=2.0 ** -14).double())) - 3).float()
    scale = (torch.round(t / step) * step).clamp(max=10240.0)
    r = torch.where(scale > 0, x.abs() / torch.where(scale > 0, scale, 1.0), 0.0)
    level = 0.5 * ((r > 0.25).float() + (r >= 0.75) + (r > 1.25) + (r >= 1.75)) + (r > 2.5).float() + (r >= 3.5) + 2.0 * (r > 5.0)
    return (level.copysign(x) * scale).flatten(-2)


def _held_key(x, code):
    """Keys (binary16) as a cache of POT4, POTM4 or INT8 holds them."""
    x = x.float()
    top = x.abs().amax(-1, keepdim=True)
    if code == INT8:
        return torch.round(x * torch.where(top > 0, 127.0 / top, 0.0)).clamp(-127, 127) * top / 127.0
    k, u = (4 if code == POTM4 else 0), (x.abs() / torch.where(top > 0, top, 1.0)).double()
    e = torch.floor(torch.log2(u.clamp(min=2.0 ** -30)))
    n = torch.floor(u * torch.exp2(k - e))                     # n <= u 2^(k - e) < n + 1
    n = n + (u * torch.exp2(k - e) >= torch.sqrt(n * (n + 1)))
    held = n * torch.exp2(e - k)
    return (torch.where(held < 2.0 ** -6, 0.0, held).float() * top).copysign(x)


def _held_value(x):
    x = x.float()
    top = x.abs().amax(-1, keepdim=True)
    g = torch.floor(torch.log2(127.0 / torch.where(top > 0, top, 1.0).double())).float()
    return torch.round(x * torch.exp2(g)) * torch.exp2(-g)


def _append_plain(s):
    case = s["case"]
    Hq, Hkv, d, code = case["q_heads"], case["kv_heads"], case["d"], case["code"]
    Q, K, V = (x.unflatten(1, (-1, d)).float() for x in s["x"].split([Hq * d, Hkv * d, Hkv * d], 1))
    angle = s["pos"].double()[:, None] * s["inv_freq"].double()                      # far positions: 64 bits
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def one(x, w):
        if case["norm"]:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w.float()
        a, b = x.unflatten(-1, (-1, 2) if case["neighbours"] else (2, -1)).unbind(-1 if case["neighbours"] else -2)
        return torch.stack([a * cos - b * sin, a * sin + b * cos], -1 if case["neighbours"] else -2).flatten(-2).half()

    Q, K, V = one(Q, s["wq"]), one(K, s["wk"]), V.half()
    if code != FP16:
        K = _rotate_hadamard(K).half() if case["hadamard"] else K
        K = _held_fp4(K) if code == FP4 else _held_key(K, code)
        K = _rotate_hadamard(K).half() if case["hadamard"] else K.half()
        V = (_held_fp4(V) if code == FP4 else _held_value(V)).half()
    s["lens"].copy_(s["lens0"] + torch.bincount(s["seq"], minlength=case["batch"]).int())
    return {"Q": Q, "K": K, "V": V, "lens": s["lens"]}


def _cache_values(s):
    """The pool as numbers: keys and values [page, 64 tokens, KV head, d] in 32 bits."""
    case, pages = s["case"], s["pages"]
    d, code, (n, H) = case["d"], case["code"], pages.shape[:2]
    half = pages.reshape(n * H * 2, -1)
    if code == FP16:
        K, V = half.view(torch.float16).reshape(-1, 2, d // 8, 32, 8).transpose(2, 3).reshape(-1, 2, 32, d).float().unbind(1)
    elif code == FP4:
        level = torch.tensor((0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0), device="cuda")
        m, h = 16 * d, len(half)
        k, a, v, c = half.split([m, m // 8, m, m // 8], 1)
        kc = torch.stack([k & 15, k >> 4], -1).reshape(h, d // 64, 2, 32, 4, 4, 2).permute(0, 3, 1, 4, 2, 5, 6).reshape(h, 32, d // 16, 16)
        ks = a.reshape(h, d // 64, 4, 8, 4).permute(0, 4, 3, 1, 2).reshape(h, 32, d // 16, 1)
        vc = torch.stack([v & 15, v >> 4], -1).reshape(h, d // 32, 8, 4, 2, 2, 2, 2, 2).permute(0, 5, 6, 3, 8, 1, 4, 7, 2).reshape(h, 32, d // 16, 16)
        vs = c.reshape(h, d // 32, 4, 2, 2, 2, 2).permute(0, 4, 6, 2, 5, 1, 3).reshape(h, 32, d // 16, 1)
        K, V = ((level[codes.int()] * (scale.to(torch.int16) << 7).view(torch.float16).float()).flatten(-2) for codes, scale in ((kc, ks), (vc, vs)))
    else:
        k, meta, v = half.split([_key_bytes(case), 128, 32 * d], 1)
        if code == POT4:
            k = torch.stack([k & 15, k >> 4], -1).reshape(-1, d // 32, 32, 32).transpose(1, 2).reshape(-1, 32, d)
        else:
            k = k.reshape(-1, d // 16, 32, 16).transpose(1, 2).reshape(-1, 32, d)
        v = v.view(torch.int8).reshape(-1, d // 16, 32, 16).transpose(1, 2).reshape(-1, 32, d)
        meta = meta.view(torch.int16)
        scale, g = meta[:, 0::2].contiguous().view(torch.float16).float()[..., None], (meta[:, 1::2] << 8 >> 8).float()[..., None]
        if code == INT8:
            K = k.view(torch.int8).float() * scale / 127.0
        else:                                                  # sign, four bits of mantissa (none), 7 - exponent (0: zero)
            e, j, sign = (k & 7).float(), (k >> 3 & 15).float() if code == POTM4 else 0.0, (k >> (7 if code == POTM4 else 3) & 1).float()
            K = torch.where(e > 0, (1.0 + j / 16.0) * torch.exp2(e - 7.0), 0.0) * (1.0 - 2.0 * sign) * scale
        V = v.float() * torch.exp2(-g)
    return [x.reshape(n, H, 64, d).transpose(1, 2) for x in (K, V)]


def _attend_plain(s):
    case = s["case"]
    Hkv, W = case["kv_heads"], case["window"]
    lens, new = _lens(case)
    Q = _rotate_hadamard(s["Q"]).half().float() if case["hadamard"] else s["Q"].float()
    if case["code"] in (POT4, POTM4, INT8):
        top = Q.abs().amax(-1, keepdim=True)
        Q = torch.round(Q * torch.where(top > 0, 127.0 / top, 0.0)).clamp(-127, 127) * (top / 127.0)
    t = torch.arange(int(lens.max()), device="cuda")
    page = s["table"][:, :(len(t) + 63) // 64].long().clamp(min=0).repeat_interleave(64, 1)[:, :len(t)]
    K, V = (x[page, t % 64] for x in _cache_values(s))         # [B, T, KV head, d]
    q = torch.zeros(case["batch"], int(new.max()), *Q.shape[1:], device="cuda")
    q[s["seq"], s["at"]] = Q
    p = torch.full(q.shape[:2], -1, device="cuda", dtype=torch.int64)                # positions of the queries; of padding: before all keys
    p[s["seq"], s["at"]] = s["pos"].long()
    seen = t <= p[..., None]
    if W:
        seen &= (t > p[..., None] - W) | (t < case["sinks"])
    z = torch.einsum("bihgd,bthd->bhgit", q.unflatten(2, (Hkv, -1)), K) / math.sqrt(case["d"])
    z = z.masked_fill_(~seen[:, None, None], -torch.inf)
    z = torch.exp_(z.sub_(z.amax(-1, keepdim=True).clamp(min=-1e30)))
    O = torch.einsum("bhgit,bthd->bihgd", z, V) / z.sum(-1).clamp(min=1e-30).permute(0, 3, 1, 2)[..., None]
    return {"O": O.flatten(2, 3)[s["seq"], s["at"]].to(TYPES[case["dtype"]])}


# ---- the same from the definitions, in 64 bits -----------------------------------------------------------------------------------------

def _exact_hadamard(x, rounded):
    """rounded: the rotation of the definition, which codes and products start from (32-bit sums of channels 1, 2, 4, ... apart, then
    binary16); otherwise in 64 bits."""
    d = x.shape[-1]
    i = torch.arange(d, device="cuda")
    x = x.float() if rounded else x.double()
    for h in (1 << k for k in range(d.bit_length() - 1)):
        x = torch.where((i & h) == 0, x + x[..., i ^ h], x[..., i ^ h] - x)
    return (x * np.float32(d ** -0.5)).half() if rounded else x / math.sqrt(d)


def _nearest(r, level, ratio):
    """The entry of the ascending table `level` that is nearest to r: in the difference (ties to the even place), or in the ratio."""
    up = torch.searchsorted(level, r.contiguous()).clamp(1, len(level) - 1)          # level[up - 1] < r <= level[up], but at the ends
    lo, hi = level[up - 1], level[up]
    if ratio:
        return torch.where(r * r >= lo * hi, hi, lo)
    return torch.where((r - lo < hi - r) | ((r - lo == hi - r) & (up % 2 == 1)), lo, hi)


def _exact_held(x, code, key):
    """The numbers that binary16 vectors are held as."""
    x = x.double()
    if code == FP16:
        return x
    if code == FP4:
        x = x.reshape(*x.shape[:-1], -1, 16)
        t = x.abs().amax(-1, keepdim=True) / 6
        step = torch.exp2(torch.floor(torch.log2(t.clamp(min=2.0 ** -14))) - 3)     # of the scales around t (rint: ties to even)
        s = torch.clamp(torch.round(t / step) * step, max=10240.0)
        r = torch.where(s > 0, x.abs() / torch.where(s > 0, s, 1.0), 0.0)
        return (torch.copysign(_nearest(r, torch.tensor((0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0), dtype=torch.float64, device="cuda"), False), x) * s).flatten(-2)
    top = x.abs().amax(-1, keepdim=True)
    if not key:
        m, e = torch.frexp(top)                                # top = m 2^e with m in [1 / 2, 1): 127 / top lies in (2^(6 - e), 2^(8 - e))
        g = 7 - e - (torch.ldexp(top, 7 - e) > 127).int()
        return torch.ldexp(torch.round(torch.ldexp(x, g)), -g)
    if code == INT8:
        step = (127.0 / top.float()).float()                   # (the decision is one of 32-bit numbers)
        return torch.round(x.float() * torch.where(top > 0, step, 0.0)).clamp(-127, 127).double() * top / 127
    k = code
    grid = torch.tensor([(1 + j / 2 ** k) * 2.0 ** -e for e in range(8, -1, -1) for j in range(2 ** k)], dtype=torch.float64, device="cuda")
    grid = grid[:len(grid) - 2 ** k + 1]                       # .. 1 is the largest
    u = _nearest(x.abs() / torch.where(top > 0, top, 1.0), grid, True)
    return torch.copysign(torch.where(u >= 2.0 ** -6, u, 0.0), x) * top


def _exact_cache(s, b, n):
    """Keys and values of n tokens of sequence b, [n, KV head, d] in 64 bits: the bytes of token t and channel c by their places in the page."""
    d, code = s["case"]["d"], s["case"]["code"]
    i = torch.arange(n, device="cuda")
    half = s["pages"][s["table"][b, i // 64].long(), :, i // 32 % 2].transpose(0, 1).long()      # [KV head, token, bytes]
    t, c = (i % 32)[:, None], torch.arange(d, device="cuda")[None]

    def byte(at):
        return half.gather(2, at.expand(len(half), n, d))

    def float16(lo):
        e, m = lo >> 10 & 31, (lo & 1023).double() / 1024
        return torch.where(e > 0, (1 + m) * torch.exp2(e.double() - 15), m * 2.0 ** -14) * (1 - 2 * (lo >> 15 & 1)).double()

    def fp4(codes, at, nibble, scale_at):
        x = byte(at) >> (4 * nibble) & 15
        f, e = x & 1, x >> 1 & 3                               # a mantissa bit, an exponent of two bits: subnormal where that is 0
        x = torch.where(e > 0, (1 + 0.5 * f.double()) * torch.exp2(e.double() - 1), 0.5 * f.double()) * (1 - 2 * (x >> 3)).double()
        return x * float16(byte(codes + scale_at) << 7)

    if code == FP16:
        at = (c // 8 * 32 + t) * 16 + c % 8 * 2
        K, V = (float16(byte(at + o) + 256 * byte(at + o + 1)) for o in (0, 64 * d))
    elif code == FP4:
        K = fp4(16 * d, (c // 64 * 2 + c // 8 % 2) * 512 + t * 16 + c % 64 // 16 * 4 + c % 8 // 2, c % 2, c // 64 * 128 + c // 16 % 4 * 32 + t % 8 * 4 + t // 8)
        v0 = 16 * d + 2 * d
        V = fp4(v0 + 16 * d, v0 + c // 32 * 512 + c % 8 * 64 + t % 8 // 2 * 16 + c // 16 % 2 * 8 + t // 16 * 4 + t // 8 % 2 * 2 + c // 8 % 2, t % 2,
                c // 32 * 64 + t % 8 // 2 * 16 + c // 16 % 2 * 8 + t // 16 * 4 + t % 2 * 2 + t // 8 % 2)
    else:
        kb = _key_bytes(s["case"])
        k = byte((c // 32 * 32 + t) * 16 + c % 32 // 2) >> (4 * (c % 2)) & 15 if code == POT4 else byte((c // 16 * 32 + t) * 16 + c % 16)
        v = byte(kb + 128 + (c // 16 * 32 + t) * 16 + c % 16)
        meta = byte(kb + 4 * t + c % 4)                                              # binary16 scale, value exponent, 0
        scale, g = float16(meta[..., 0:1] + 256 * meta[..., 1:2]), meta[..., 2:3]
        if code == INT8:
            K = (k - 256 * (k >> 7)).double() * scale / 127
        else:
            j, sign = ((k >> 3 & 15).double() / 16, k >> 7) if code == POTM4 else (0.0, k >> 3)
            K = torch.where(k & 7 > 0, (1 + j) * torch.exp2((k & 7).double() - 7), 0.0) * (1 - 2 * sign).double() * scale
        V = (v - 256 * (v >> 7)).double() * torch.exp2(-(g - 256 * (g >> 7)).double())
    return K.transpose(0, 1), V.transpose(0, 1)


def _exact_attend(s):
    case = s["case"]
    lens, new = _lens(case)
    d, W, O = case["d"], case["window"], []
    for b, (n, m) in enumerate(zip(lens, new)):
        K, V = _exact_cache(s, b, int(n))
        Q = s["Q"][s["cu"][b]:s["cu"][b + 1]]
        q = (_exact_hadamard(Q, True) if case["hadamard"] else Q).float()
        if case["code"] in (POT4, POTM4, INT8):                # (the decision is one of 32-bit numbers)
            top = q.abs().amax(-1, keepdim=True)
            q = torch.round(q * torch.where(top > 0, 127.0 / top, 0.0)).clamp(-127, 127).double() * top.double() / 127
        i, j = torch.arange(int(n - m), int(n), device="cuda")[:, None], torch.arange(int(n), device="cuda")[None]
        hidden = j > i
        if W:
            hidden = hidden | ((i - j >= W) & (j >= case["sinks"]))
        heads = [torch.softmax((q[:, h].double() @ K[:, h * case["kv_heads"] // case["q_heads"]].T / math.sqrt(d)).masked_fill_(hidden, -torch.inf), -1)
                 @ V[:, h * case["kv_heads"] // case["q_heads"]] for h in range(case["q_heads"])]
        O.append(torch.stack(heads, 1))
    return {"O": torch.cat(O)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] != "append":
        return _exact_attend(s)
    Hq, Hkv, d = case["q_heads"], case["kv_heads"], case["d"]
    x = s["x"].double().reshape(len(s["x"]), -1, d)
    y = x[:, :Hq + Hkv].clone()
    if case["norm"]:
        y = y / torch.sqrt((y ** 2).mean(-1, keepdim=True) + 1e-6) * torch.cat([s["wq"].double().expand(Hq, d), s["wk"].double().expand(Hkv, d)])
    j = torch.arange(d // 2, device="cuda")
    first, second = (2 * j, 2 * j + 1) if case["neighbours"] else (j, j + d // 2)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["pos"].double()[:, None] * s["inv_freq"].double())
    z = torch.complex(y[..., first], y[..., second]) * turn[:, None]
    y[..., first], y[..., second] = z.real, z.imag
    K = y[:, Hq:].half()                                       # the cache's codes are those of the binary16 numbers
    K = _exact_held(_exact_hadamard(K, True) if case["hadamard"] else K, case["code"], True)
    return {"Q": y[:, :Hq], "K": _exact_hadamard(K, False) if case["hadamard"] else K, "V": _exact_held(x[:, Hq + Hkv:].half(), case["code"], False),
            "lens": s["lens0"] + torch.from_numpy(np.diff(s["cu"])).int().cuda()}


def work(case):
    """Every input read once, every output written once: projections, codes in and out and rows of the new tokens; or the keys that one of the queries sees, queries and outputs.
    4 operations per query head, visible key and channel, 8 per rotated channel."""
    d, Hq, Hkv, W, k = case["d"], case["q_heads"], case["kv_heads"], case["window"], case["sinks"]
    lens, new = _lens(case)
    n, record = int(new.sum()), _half_bytes(case) // 32
    if case["kind"] == "append":
        size = (2, 2, 4)[case["dtype"]]
        return {"bytes": n * ((Hq + 2 * Hkv) * d * (size + 2) + 2 * Hkv * record + 4), "flops": 8 * n * (Hq + Hkv) * d}
    keys = pairs = 0
    for t, m in zip(lens.tolist(), new.tolist()):
        p = np.arange(t - m, t)
        seen = np.minimum(p + 1, W) + np.minimum(np.maximum(p + 1 - W, 0), k) if W else p + 1
        pairs += int(seen.sum())
        keys += min(t, m - 1 + W + min(k, max(0, t - m + 1 - W))) if W else t
    return {"bytes": keys * Hkv * record + n * Hq * d * 4, "flops": 4 * pairs * Hq * d}
