"""Timed cases of the operators around the 4-bit cache: what turns a layer's projections into queries, keys and values
(``rotate_qkv``), the cache with keys and values in 4 bits (``fill_kv``, ``decode_attention``, ``decode_step`` with ``SA_KV_FP4``)
and the way back out of a cache (``read_kv``).

Kinds of case:

  rotate     norms of queries and keys for each head, rotation by the token's position(s), values converted: one layer
  fill_read  the keys and values of prompts into a 4-bit cache and back out as binary16
  read       keys and values of a cache that is already there, back out as binary16
  decode     one decode-attention call over a 4-bit cache (one layer)
  step       one decode step over a 4-bit cache (append the new token and attend), and the new token as the cache holds it

Shapes: 32 query / 4 KV heads of 64 channels, 32 / 8 heads of 128, and the odd ones between, from one token to 32 sequences of 32 768.

4-bit cache.  A vector of d channels is cut into blocks of 16.  A block's scale is s = max|x| / 6 rounded to an unsigned 8-bit float (5
exponent, 3 mantissa bits; nearest, ties to even; at most 10240), held as a byte b with s = binary16 pattern b << 7.  A channel's code is
x / s rounded to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (ties to the even code, 6 at most), the sign in bit 3.  The value it stands for is
code * s.  A page of one KV head holds 64 tokens as two halves; in a half of 32 tokens:
  key codes     [d / 32 chunks][32 tokens][16 bytes]: word i of chunk c holds channels 64 (c / 2) + 16 i + 8 (c % 2) .. + 7, two a byte
  key scales    [d / 64][block % 4][token % 8][token / 8]
  value codes   [d / 32][channel % 8][token % 8 / 2][channel / 16 % 2][token / 16][token / 8 % 2][channel / 8 % 2], a byte: tokens 2 i, 2 i + 1
  value scales  [d / 32][token % 8 / 2][channel / 16 % 2][token / 16][token % 2][token / 8 % 2]
"""
import math

import numpy as np
import torch

own = False                              # set by who times: False: elementary torch operations, True: the library's kernels

POTM4, INT8, FP4 = 4, 8, 32              # codes of a cache
F16, BF16, F32 = 0, 1, 2                 # types of a projection's output
TYPES = (torch.float16, torch.bfloat16, torch.float32)
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _case(kind, *, d=64, q_heads=32, kv_heads=4, batch=1, tokens=1024, shortest=0, code=FP4, hadamard=False, dtype=BF16, norm=True, rotary=0,
          neighbours=False, axes=1, **more):
    """tokens: length of every sequence, or the longest of a ragged batch whose shortest is `shortest` (0: all equal); kind rotate:
    tokens in all.  rotary: channels that are rotated (0: all).  neighbours: channels 2 j, 2 j + 1 form a pair, not j, j + rotary / 2."""
    return dict(more, kind=kind, d=d, q_heads=q_heads, kv_heads=kv_heads, batch=batch, tokens=tokens, shortest=shortest, code=code,
                hadamard=hadamard, dtype=dtype, norm=norm, rotary=rotary or d, neighbours=neighbours, axes=axes)


def listed():
    return [
        # a token of one sequence: the smallest call
        _case("rotate", tokens=1, dtype=F16, norm=False, name="rotate_token"),
        # a prompt of a model with norms of queries and keys
        _case("rotate", d=128, kv_heads=8, tokens=8192, name="rotate_prompt_8k"),
        # images and video: time, height and width, FP32 projections, a part of the channels rotated
        _case("rotate", d=128, q_heads=16, kv_heads=16, tokens=5001, dtype=F32, rotary=96, neighbours=True, axes=3, name="rotate_3axes_5001"),
        # prompts of four sequences into the cache, and out again for the next chunk's attention
        _case("fill_read", batch=4, tokens=8192, shortest=1000, name="fill_read_b4_8k"),
        # one prompt that fills no page, rotated keys
        _case("fill_read", d=128, kv_heads=8, tokens=20001, hadamard=True, name="fill_read_d128_20001"),
        # a power-of-two cache whose contents move on to another form
        _case("read", batch=8, tokens=16384, code=POTM4, name="read_potm4_b8_16k"),
        # attention of one token over a short context: latency
        _case("decode", q_heads=8, kv_heads=1, tokens=1024, name="decode_1k"),
        # continuous batching: 16 sequences of mixed lengths
        _case("decode", batch=16, tokens=16384, shortest=2048, name="decode_ragged_b16"),
        # one very long document
        _case("decode", d=128, kv_heads=8, tokens=131072, hadamard=True, name="decode_d128_128k"),
        # the largest: 32 sequences of 32k tokens
        _case("decode", batch=32, tokens=32768, name="decode_b32_32k"),
        # a decode step of one chat
        _case("step", tokens=4095, name="step_b1_4095"),
        # a decode step of a large batch of ordinary contexts
        _case("step", d=128, kv_heads=8, batch=32, tokens=4096, name="step_d128_b32_4k"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "rotate", "fill_read", "read", "decode", "decode", "decode", "step", "step"])
    d, q_heads, kv_heads = rng.choice([(64, 32, 4), (64, 32, 4), (128, 32, 8), (64, 8, 2), (64, 1, 1), (128, 16, 16), (128, 40, 8), (64, 12, 1)])
    if kind == "rotate":
        rotary = rng.choice([d, d, d // 2, d - 16])
        return _case(kind, d=d, q_heads=q_heads, kv_heads=kv_heads, tokens=_log_int(rng, 1, 2 ** 26 // (d * (q_heads + 2 * kv_heads))),
                     dtype=rng.choice([F16, BF16, F32]), norm=rng.random() < 0.6, rotary=rotary, neighbours=rng.random() < 0.4, axes=rng.choice([1, 1, 2, 3, 4]))
    batch = rng.choice([1, 1, 2, 3, 4, 8, 13, 16, 32])
    most = 32 * 32768 * 4 * 64 // (batch * kv_heads * d)       # at most the cached keys of the largest listed case, or an eighth of them
    most = min(most if kind == "decode" else most // 8, 131072 if batch == 1 else 32768)
    tokens = _log_int(rng, 100, max(400, most))
    shortest = max(1, tokens // rng.choice([2, 8])) if batch > 1 and rng.random() < 0.5 else 0
    return _case(kind, d=d, q_heads=q_heads, kv_heads=kv_heads, batch=batch, tokens=tokens, shortest=shortest,
                 code=rng.choice([POTM4, INT8, FP4]) if kind == "read" else FP4, hadamard=kind != "read" and rng.random() < 0.3)


def _lens(case):
    """Cached tokens per sequence: all equal, or spread evenly from the shortest to the longest in a mixed order."""
    B, T, lo = case["batch"], case["tokens"], case["shortest"]
    if not lo or B == 1:
        return np.full(B, T, dtype=np.int64)
    steps = np.linspace(lo, T, B).astype(np.int64)
    return steps[(np.arange(B) * 7 + 3) % B] if B % 7 else steps[::-1].copy()


# ---- inputs -------------------------------------------------------------------------------------------------------------------------

def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _codes(x):
    """[..., d] binary16 -> codes [..., d] and scale bytes [..., d / 16], both uint8.  The decisions are exact in 32 bits: a quotient of a
    binary16 number by 6 or by a scale of 4 bits that is no tie lies further from one than 32 bits round it."""
    x = x.float().unflatten(-1, (-1, 16))
    t = x.abs().amax(-1) / 6.0
    u = t.view(torch.int32)
    b = torch.where(t >= 2.0 ** -14, ((u + 0x7ffff + ((u >> 20) & 1)) >> 20) - (112 << 3), torch.round(t * 2.0 ** 17).int()).clamp(max=0xe2)
    s = _scales(b)[..., None]
    r = torch.where(s > 0, x.abs() / torch.where(s > 0, s, 1.0), 0.0)
    code = (r > 0.25).byte() + (r >= 0.75) + (r > 1.25) + (r >= 1.75) + (r > 2.5) + (r >= 3.5) + (r > 5.0)
    return (code + 8 * ((x < 0) & (code > 0))).byte().flatten(-2), b.byte()


def _scales(b):
    return (b.to(torch.int16) << 7).view(torch.float16).float()


def _values(codes, b):
    level = torch.tensor(LEVELS + tuple(-x for x in LEVELS), device=codes.device)
    return (level[codes.int()].unflatten(-1, (-1, 16)) * _scales(b)[..., None]).flatten(-2)


def _pack(kc, ks, vc, vs):
    """Codes [n, 32, d] and scale bytes [n, 32, d / 16] of n half pages -> the half pages [n, bytes]."""
    n, d = len(kc), kc.shape[-1]
    k = kc.reshape(n, 32, d // 64, 4, 2, 4, 2).permute(0, 2, 4, 1, 3, 5, 6).reshape(n, -1, 2)
    a = ks.reshape(n, 4, 8, d // 64, 4).permute(0, 3, 4, 2, 1).reshape(n, -1)
    v = vc.reshape(n, 2, 2, 4, 2, d // 32, 2, 2, 8).permute(0, 5, 8, 3, 6, 1, 2, 7, 4).reshape(n, -1, 2)
    c = vs.reshape(n, 2, 2, 4, 2, d // 32, 2).permute(0, 5, 3, 6, 1, 4, 2).reshape(n, -1)
    return torch.cat([k[..., 0] | (k[..., 1] << 4), a, v[..., 0] | (v[..., 1] << 4), c], 1)


def _unpack(half, d):
    """Half pages [n, bytes] -> codes and scale bytes of keys and values, as _pack takes them."""
    n, m = len(half), 16 * d
    k, a, v, c = half.split([m, m // 8, m, m // 8], 1)
    kc = torch.stack([k & 15, k >> 4], -1).reshape(n, d // 64, 2, 32, 4, 4, 2).permute(0, 3, 1, 4, 2, 5, 6).reshape(n, 32, d)
    ks = a.reshape(n, d // 64, 4, 8, 4).permute(0, 4, 3, 1, 2).reshape(n, 32, d // 16)
    vc = torch.stack([v & 15, v >> 4], -1).reshape(n, d // 32, 8, 4, 2, 2, 2, 2, 2).permute(0, 5, 6, 3, 8, 1, 4, 7, 2).reshape(n, 32, d)
    vs = c.reshape(n, d // 32, 4, 2, 2, 2, 2).permute(0, 4, 6, 2, 5, 1, 3).reshape(n, 32, d // 16)
    return kc, ks, vc, vs


def _half_bytes(case):
    d = case["d"]
    return 32 * (d + d // 8 if case["code"] == FP4 else 2 * d + 4)


def _pages(case, gen, n_pages):
    """A pool of full pages: [page, KV head, half, bytes]."""
    H, d = case["kv_heads"], case["d"]
    n = n_pages * H * 2
    if case["code"] == FP4:
        K = (_normal(gen, n, 32, d) * torch.exp(0.5 * _normal(gen, 1, 1, d))).half()
        half = _pack(*_codes(K), *_codes(_normal(gen, n, 32, d).half()))
    else:
        half = torch.randint(0, 256, (n, _half_bytes(case)), generator=gen, device="cuda", dtype=torch.uint8)
        if case["code"] == POTM4:                              # (an exponent field of 0 is the zero code)
            half[:, :32 * d].mul_((half[:, :32 * d] & 7) > 0)
        meta = half[:, 32 * d:32 * d + 128].view(torch.int16)                        # scale of the key, exponent of the value's scale
        meta[:, 0::2] = (1.0 + _normal(gen, n, 32).abs()).half().view(torch.int16)
        meta[:, 1::2] = torch.randint(4, 7, (n, 32), generator=gen, device="cuda").short()
    return half.reshape(n_pages, H, 2, -1)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    B, Hq, Hkv, d, kind = case["batch"], case["q_heads"], case["kv_heads"], case["d"], case["kind"]
    s = dict(case=case)
    if kind == "rotate":
        n, t, R = case["tokens"], TYPES[case["dtype"]], case["rotary"]
        s["x"] = _normal(gen, n, (Hq + 2 * Hkv) * d).to(t)                           # queries, keys and values of a token side by side
        i = torch.arange(n, device="cuda")
        grid = torch.stack([i // 1024, i // 32 % 32, i % 32, i])[:case["axes"]] if case["axes"] > 1 else i[None]
        s["pos"] = (grid + torch.randint(0, 131072 - n, (1, 1), generator=gen, device="cuda")).int().contiguous()
        s["inv_freq"] = (10000.0 ** (-torch.arange(R // 2, device="cuda", dtype=torch.float64) * 2 / R)).float()
        s["axis"] = (torch.arange(R // 2, device="cuda") * case["axes"] // (R // 2)).byte()
        s["wq"], s["wk"] = ((1.0 + 0.2 * _normal(gen, d)).to(t) if case["norm"] else None for _ in "qk")
        s["Q"], s["K"], s["V"] = (torch.zeros(n, h, d, dtype=torch.float16, device="cuda") for h in (Hq, Hkv, Hkv))
    else:
        lens = _lens(case)
        pages = np.maximum((lens + (1 if kind == "step" else 0) + 63) // 64, 1)
        table = np.full((B, int(pages.max())), -1, dtype=np.int32)
        table[np.arange(table.shape[1])[None] < pages[:, None]] = np.random.Generator(np.random.PCG64(seed)).permutation(int(pages.sum()))
        n = B if kind == "step" else int(lens.sum())
        s["cu"] = np.concatenate([[0], np.cumsum(np.ones_like(lens) if kind == "step" else lens)])
        s["lens0"] = torch.from_numpy(lens.astype(np.int32)).cuda()
        s["lens"] = s["lens0"].clone()
        s["start"] = lens if kind == "step" else np.zeros_like(lens)
        s["table"] = torch.from_numpy(table).cuda()
        s["pages"] = (torch.zeros(int(pages.sum()), Hkv, 2, _half_bytes(case), dtype=torch.uint8, device="cuda") if kind == "fill_read"
                      else _pages(case, gen, int(pages.sum())))
        if kind in ("fill_read", "step"):
            s["K_new"] = (_normal(gen, n, Hkv, d) * torch.exp(0.5 * _normal(gen, 1, Hkv, d))).half()
            s["V_new"] = _normal(gen, n, Hkv, d).half()
        if kind in ("decode", "step"):
            s["Q"] = _normal(gen, B, Hq, d).half()
            s["O"] = torch.zeros(B, Hq, d, dtype=torch.float32, device="cuda")
        if kind != "decode":
            s["K"], s["V"] = (torch.zeros(n, Hkv, d, dtype=torch.float16, device="cuda") for _ in "kv")
    if own:
        _handles(s)
    torch.cuda.synchronize()
    return s


def _handles(s):
    """What a program keeps from call to call: the configuration, the cache's handle and workspace, the rotation's tables."""
    from paper_2609_09208_b200 import binding as sa
    case = s["case"]
    s["sa"] = sa
    s["cfg"] = sa.make_config(case["d"], case["q_heads"], case["kv_heads"], case["code"], hadamard=case["hadamard"])
    if case["kind"] == "rotate":
        s["rotary"] = sa.Rotary(s["cfg"], s["inv_freq"], dtype=TYPES[case["dtype"]], pairs="neighbours" if case["neighbours"] else "halves",
                                n_axes=case["axes"], pair_axis=s["axis"], norm=case["norm"], eps=1e-6, q_weight=s["wq"], k_weight=s["wk"])
        Hq, Hkv, d = case["q_heads"], case["kv_heads"], case["d"]
        s["qkv"] = [x.unflatten(1, (-1, d)) for x in s["x"].split([Hq * d, Hkv * d, Hkv * d], 1)]
        return
    s["handle"] = sa.make_cache(s["pages"], s["table"], s["lens"], len(s["pages"]))
    s["workspace"] = torch.empty(max(16, sa.workspace_bytes(s["cfg"], *s["table"].shape)), dtype=torch.uint8, device="cuda")


# ---- the operators ------------------------------------------------------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    sa, kind = s["sa"], s["case"]["kind"]
    if kind == "rotate":
        sa.rotate_qkv(s["rotary"], *s["qkv"], s["pos"], s["Q"], s["K"], s["V"])
        return {"Q": s["Q"], "K": s["K"], "V": s["V"]}
    cfg, cache = s["cfg"], s["handle"]
    if kind == "decode":
        sa.decode_attention(cfg, cache, s["Q"], s["O"], s["workspace"])
        return {"O": s["O"]}
    if kind == "fill_read":
        sa.fill_kv(cfg, cache, s["K_new"], s["V_new"], s["cu"])
    if kind == "step":
        s["lens"].copy_(s["lens0"])                            # as a program does that drops a rejected token
        sa.decode_step(cfg, cache, s["Q"], s["K_new"], s["V_new"], s["O"], s["workspace"])
    sa.read_kv(cfg, cache, s["start"], s["cu"], s["K"], s["V"])
    return {"K": s["K"], "V": s["V"], **({"O": s["O"], "lens": s["lens"]} if kind == "step" else {})}


def _rotate_hadamard(x):
    """Walsh-Hadamard rotation of the last axis, in 32 bits, in the order that the cache's definition fixes; rounded to binary16."""
    x, d = x.float(), x.shape[-1]
    for h in (1 << i for i in range(d.bit_length() - 1)):
        a, b = x.unflatten(-1, (-1, 2, h)).unbind(-2)
        x = torch.stack([a + b, a - b], -2).flatten(-3)
    return (x * torch.tensor(1.0 / math.sqrt(d), dtype=torch.float32)).half()


def _tokens(s, lens):
    """Places of the tokens of the sequences, [B, T] each: pool page and slot; and which of them there are."""
    i = torch.arange(int(lens.max()), device="cuda")[None]
    there = i < torch.from_numpy(lens).cuda()[:, None]
    return s["table"][:, :(int(lens.max()) + 63) // 64].long().repeat_interleave(64, 1)[:, :i.shape[1]], i % 64, there


def _cache_values(s):
    """The pool as numbers: keys and values [page, 64 tokens, KV head, d] in 32 bits."""
    case, pages = s["case"], s["pages"]
    d, (n, H) = case["d"], pages.shape[:2]
    half = pages.reshape(n * H * 2, -1)
    if case["code"] == FP4:
        kc, ks, vc, vs = _unpack(half, d)
        K, V = _values(kc, ks), _values(vc, vs)
    else:
        k, meta, v = half.split([32 * d, 128, 32 * d], 1)
        k, v = (x.reshape(-1, d // 16, 32, 16).transpose(1, 2).reshape(-1, 32, d) for x in (k, v.view(torch.int8)))
        meta = meta.view(torch.int16)
        scale, g = meta[:, 0::2].contiguous().view(torch.float16).float()[..., None], (meta[:, 1::2] << 8 >> 8).float()[..., None]
        if case["code"] == INT8:
            K = k.view(torch.int8).float() * scale / 127.0
        else:                                                  # sign, four bits of mantissa, 7 - exponent (0: zero)
            e = (k & 7).float()
            K = torch.where(e > 0, (1.0 + ((k >> 3) & 15).float() / 16.0) * torch.exp2(e - 7.0), 0.0) * torch.where(k >= 128, -1.0, 1.0) * scale
        V = v.float() * torch.exp2(-g)
    return [x.reshape(n, H, 64, d).transpose(1, 2) for x in (K, V)]


def _append_plain(s):
    """The new token of every sequence into its half page."""
    d, at = s["case"]["d"], s["lens0"].long()
    page = s["table"].gather(1, (at // 64)[:, None])[:, 0].long()
    K = _rotate_hadamard(s["K_new"]) if s["case"]["hadamard"] else s["K_new"]
    half = s["pages"][page, :, at % 64 // 32]                  # [B, KV head, bytes]
    parts = [x.clone() for x in _unpack(half.flatten(0, 1), d)]
    row, t = torch.arange(len(parts[0]), device="cuda"), (at % 32).repeat_interleave(half.shape[1])
    for part, new in zip(parts, (*_codes(K), *_codes(s["V_new"]))):
        part[row, t] = new.flatten(0, 1)
    s["pages"][page, :, at % 64 // 32] = _pack(*parts).reshape(half.shape)


def _attend_plain(s, lens):
    case = s["case"]
    page, slot, there = _tokens(s, lens)
    K, V = (x[page, slot] for x in _cache_values(s))          # [B, T, KV head, d]
    Q = (_rotate_hadamard(s["Q"]) if case["hadamard"] else s["Q"]).float().unflatten(1, (case["kv_heads"], -1))
    z = torch.einsum("bhgd,bthd->bhgt", Q, K) / math.sqrt(case["d"])
    p = torch.exp(z - z.masked_fill(~there[:, None, None], -torch.inf).amax(-1, keepdim=True)) * there[:, None, None]
    return (torch.einsum("bhgt,bthd->bhgd", p, V) / p.sum(-1, keepdim=True)).flatten(1, 2)


def _rotate_plain(s):
    case = s["case"]
    Hq, Hkv, d, R = case["q_heads"], case["kv_heads"], case["d"], case["rotary"]
    Q, K, V = (x.unflatten(1, (-1, d)).float() for x in s["x"].split([Hq * d, Hkv * d, Hkv * d], 1))
    angle = s["pos"][s["axis"].long()].double().T * s["inv_freq"].double()           # far positions: 64 bits
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def one(x, w):
        if case["norm"]:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w.float()
        pairs = x[..., :R].unflatten(-1, (-1, 2) if case["neighbours"] else (2, -1))
        a, b = pairs.unbind(-1 if case["neighbours"] else -2)
        y = torch.stack([a * cos - b * sin, a * sin + b * cos], -1 if case["neighbours"] else -2).flatten(-2)
        return torch.cat([y, x[..., R:]], -1).half()

    return {"Q": one(Q, s["wq"]), "K": one(K, s["wk"]), "V": V.half()}


def _run_plain(s):
    case, kind = s["case"], s["case"]["kind"]
    if kind == "rotate":
        return _rotate_plain(s)
    lens = _lens(case)
    if kind == "decode":
        return {"O": _attend_plain(s, lens)}
    if kind == "step":
        _append_plain(s)
        O = _attend_plain(s, lens + 1)
        s["lens"].copy_(s["lens0"] + 1)
    if kind == "fill_read":                                    # whole half pages: what lies behind a sequence's end is zero
        there = torch.arange(s["table"].shape[1] * 64, device="cuda")[None] < s["lens0"][:, None]
        row = torch.where(there, (there.flatten().cumsum(0) - 1).view_as(there), 0)
        new = (_rotate_hadamard(s["K_new"]) if case["hadamard"] else s["K_new"]), s["V_new"]
        mapped = s["table"] >= 0
        parts = [c.unflatten(1, (-1, 2, 32)).permute(0, 1, 4, 2, 3, 5)[mapped].flatten(0, 2)
                 for x in new for c in _codes(torch.where(there[..., None, None], x[row], 0.0).half())]
        s["pages"][s["table"][mapped].long()] = _pack(*parts).reshape(-1, *s["pages"].shape[1:])
    if kind == "step":                                         # the one token of every sequence
        at = s["lens0"].long()
        K, V = (x[s["table"].gather(1, (at // 64)[:, None])[:, 0].long(), at % 64] for x in _cache_values(s))
    else:
        page, slot, there = _tokens(s, lens)
        K, V = (x[page[there], slot.expand_as(page)[there]] for x in _cache_values(s))
    K = _rotate_hadamard(K) if case["hadamard"] else K.half()
    return {"K": K, "V": V.half(), **({"O": O, "lens": s["lens"]} if kind == "step" else {})}


# ---- the same from the definitions, in 64 bits -----------------------------------------------------------------------------------------

def _exact_codes(x):
    """The numbers that binary16 vectors are held as."""
    level = torch.tensor(LEVELS, dtype=torch.float64, device="cuda")
    x = x.double().reshape(*x.shape[:-1], -1, 16)
    t = x.abs().amax(-1, keepdim=True) / 6
    step = torch.exp2(torch.floor(torch.log2(t.clamp(min=2.0 ** -14))) - 3)         # of the scales around t (rint: ties to even)
    s = torch.clamp(torch.round(t / step) * step, max=10240.0)
    r = torch.where(s > 0, x.abs() / torch.where(s > 0, s, 1.0), 0.0)
    up = torch.searchsorted(level, r.contiguous()).clamp(1, 7)                      # level[up - 1] < r <= level[up], but at the ends
    lo, hi = level[up - 1], level[up]
    nearer = torch.where((r - lo < hi - r) | ((r - lo == hi - r) & (up % 2 == 1)), lo, hi)
    return (torch.copysign(nearer, x) * s).flatten(-2)


def _exact_hadamard(x, rounded):
    """rounded: the rotation of the definition, which codes and products start from (32-bit sums of channels 1, 2, 4, ... apart, then
    binary16); otherwise in 64 bits."""
    d = x.shape[-1]
    i = torch.arange(d, device="cuda")
    x = x.float() if rounded else x.double()
    for h in (1 << k for k in range(d.bit_length() - 1)):
        x = torch.where((i & h) == 0, x + x[..., i ^ h], x[..., i ^ h] - x)
    return (x * np.float32(d ** -0.5)).half() if rounded else x / math.sqrt(d)


def _exact_cache(s, b, n):
    """Keys and values of n tokens of sequence b, [n, KV head, d] in 64 bits: the bytes of token t and channel c by their places in the page."""
    d, code = s["case"]["d"], s["case"]["code"]
    i = torch.arange(n, device="cuda")
    half = s["pages"][s["table"][b, i // 64].long(), :, i // 32 % 2].transpose(0, 1).long()      # [KV head, token, bytes]
    t, c = (i % 32)[:, None], torch.arange(d, device="cuda")[None]

    def byte(at):
        return half.gather(2, at.expand(len(half), n, d))

    def fp4(codes, at, nibble, scale_at):
        x = byte(at) >> (4 * nibble) & 15
        f, e = x & 1, x >> 1 & 3                               # a mantissa bit, an exponent of two bits: subnormal where that is 0
        x = torch.where(e > 0, (1 + 0.5 * f.double()) * torch.exp2(e.double() - 1), 0.5 * f.double()) * (1 - 2 * (x >> 3)).double()
        b = byte(codes + scale_at)
        return x * torch.where(b >> 3 > 0, (1 + (b & 7).double() / 8) * torch.exp2((b >> 3).double() - 15), (b & 7).double() * 2.0 ** -17)

    if code == FP4:
        K = fp4(16 * d, (c // 64 * 2 + c // 8 % 2) * 512 + t * 16 + c % 64 // 16 * 4 + c % 8 // 2, c % 2, c // 64 * 128 + c // 16 % 4 * 32 + t % 8 * 4 + t // 8)
        v0 = 16 * d + 2 * d
        V = fp4(v0 + 16 * d, v0 + c // 32 * 512 + c % 8 * 64 + t % 8 // 2 * 16 + c // 16 % 2 * 8 + t // 16 * 4 + t // 8 % 2 * 2 + c // 8 % 2, t % 2,
                c // 32 * 64 + t % 8 // 2 * 16 + c // 16 % 2 * 8 + t // 16 * 4 + t % 2 * 2 + t // 8 % 2)
        return K.transpose(0, 1), V.transpose(0, 1)
    at = c // 16 * 512 + t * 16 + c % 16
    k, v = byte(at), byte(32 * d + 128 + at)
    meta = byte(32 * d + 4 * t + torch.arange(d, device="cuda")[None] % 4)                       # binary16 scale, value exponent, 0
    lo = meta[..., 0:1] + 256 * meta[..., 1:2]
    scale = torch.where(lo >> 10 > 0, (1 + (lo & 1023).double() / 1024) * torch.exp2((lo >> 10).double() - 15), (lo & 1023).double() * 2.0 ** -24)
    if code == INT8:
        K = (k - 256 * (k >> 7)).double() * scale / 127
    else:
        K = torch.where(k & 7 > 0, (1 + (k >> 3 & 15).double() / 16) * torch.exp2((k & 7).double() - 7), 0.0) * (1 - 2 * (k >> 7)).double() * scale
    g = meta[..., 2:3]
    V = (v - 256 * (v >> 7)).double() * torch.exp2(-(g - 256 * (g >> 7)).double())
    return K.transpose(0, 1), V.transpose(0, 1)


def exact(case, seed):
    s = prepare(case, seed)
    kind, d, had = case["kind"], case["d"], case["hadamard"]
    if kind == "rotate":
        Hq, Hkv, R = case["q_heads"], case["kv_heads"], case["rotary"]
        x = s["x"].double().reshape(len(s["x"]), -1, d)
        y = x.clone()
        if case["norm"]:
            w = torch.cat([s["wq"].double().expand(Hq, d), s["wk"].double().expand(Hkv, d)])
            y[:, :Hq + Hkv] = x[:, :Hq + Hkv] / torch.sqrt((x[:, :Hq + Hkv] ** 2).mean(-1, keepdim=True) + 1e-6) * w
        j = torch.arange(R // 2, device="cuda")
        first, second = (2 * j, 2 * j + 1) if case["neighbours"] else (j, j + R // 2)
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["pos"].double()[s["axis"].long(), :].T * s["inv_freq"].double())
        z = torch.complex(y[:, :Hq + Hkv, first], y[:, :Hq + Hkv, second]) * turn[:, None]
        y[:, :Hq + Hkv, first], y[:, :Hq + Hkv, second] = z.real, z.imag
        return {"Q": y[:, :Hq], "K": y[:, Hq:Hq + Hkv], "V": y[:, Hq + Hkv:]}
    lens, out = _lens(case), {}
    if kind in ("fill_read", "step"):
        K = _exact_codes(_exact_hadamard(s["K_new"], True) if had else s["K_new"])
        out = {"K": _exact_hadamard(K, False) if had else K, "V": _exact_codes(s["V_new"])}
    if kind == "read":
        both = [_exact_cache(s, b, int(n)) for b, n in enumerate(lens)]
        out = {"K": torch.cat([k for k, _ in both]), "V": torch.cat([v for _, v in both])}
    if kind in ("decode", "step"):
        O = []
        for b, n in enumerate(lens):
            Kb, Vb = _exact_cache(s, b, int(n))
            if kind == "step":
                Kb, Vb = torch.cat([Kb, K[b:b + 1]]), torch.cat([Vb, out["V"][b:b + 1]])
            q = (_exact_hadamard(s["Q"][b], True) if had else s["Q"][b]).double().reshape(case["kv_heads"], -1, d)
            O.append((torch.softmax(q @ Kb.permute(1, 2, 0) / math.sqrt(d), -1) @ Vb.transpose(0, 1)).reshape(-1, d))
        out["O"] = torch.stack(O)
    if kind == "step":
        out["lens"] = s["lens0"] + 1
    return out


def work(case):
    """Every input read once, every output written once; 4 operations per query head, key and dimension, 8 per rotated channel."""
    d, Hq, Hkv, B, n = case["d"], case["q_heads"], case["kv_heads"], case["batch"], int(_lens(case).sum())
    record = _half_bytes(case) // 32
    if case["kind"] == "rotate":
        n, size = case["tokens"], (2, 2, 4)[case["dtype"]]
        return {"bytes": n * (Hq + 2 * Hkv) * d * (size + 2) + 4 * n * case["axes"], "flops": 8 * n * (Hq + Hkv) * d}
    if case["kind"] == "fill_read":
        return {"bytes": 2 * n * Hkv * (4 * d + record), "flops": 0}
    if case["kind"] == "read":
        return {"bytes": n * Hkv * (4 * d + record), "flops": 0}
    new = B if case["kind"] == "step" else 0
    return {"bytes": n * Hkv * record + B * Hq * d * 6 + new * Hkv * (8 * d + 2 * record), "flops": 4 * (n + new) * Hq * d}
