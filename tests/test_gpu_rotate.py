"""sa_rotate_qkv: norms of queries and keys, position rotation, conversion, against the formulas in 64 bits; and a run of it with the
cache, steps and reads behind it."""
import numpy as np
import pytest

import fp4_reference as fp4
from paper_2609_09208_b200 import binding as sa
from paper_2609_09208_b200 import build as sa_build
from paper_2609_09208_b200 import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    sa_build.build()


def frequencies(R, base=10000.0):
    return (base ** (-np.arange(R // 2) * 2.0 / R)).astype(np.float32)


def reference(x, R, neighbours, pos, axis, inv_freq, norm, eps, w, scale):
    """x [n, H, d] float64 -> the operator's definition, and the magnitudes that its roundings are relative to."""
    y = x.copy()
    if norm:
        y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (1.0 if w is None else w)
    size = np.abs(y)
    if R:
        angle = pos[axis].astype(np.float64).T * inv_freq.astype(np.float64)               # [n, R / 2]
        c, s = scale * np.cos(angle)[:, None], scale * np.sin(angle)[:, None]
        j = np.arange(R // 2)
        a, b = (2 * j, 2 * j + 1) if neighbours else (j, j + R // 2)
        p, q = y[..., a].copy(), y[..., b].copy()
        y[..., a], y[..., b] = p * c - q * s, p * s + q * c
        size[..., a] = size[..., b] = scale * (np.abs(p) + np.abs(q))
    return y, size


def tolerance(y, size):
    """One rounding to binary16, and 32-bit roundings before it: a norm's sum of up to 128 squares and its root (70 of 2^-24 relative at most),
    three products, the turn's sine and cosine (an angle in 64 bits, 2^-22 of a turn's length and the function's 2 units) and the rotation's."""
    return np.maximum(np.abs(y) * 2.0 ** -11, 2.0 ** -25) * (1 + 2.0 ** -10) + 90 * 2.0 ** -24 * size


CASES = [
    # d, Hq, Hkv, type, R, neighbours, axes, norm, weights, scale, tokens
    (64, 32, 4, "float16", 64, False, 1, False, False, 1.0, 1), (64, 32, 4, "bfloat16", 64, False, 1, True, True, 1.0, 7),
    (128, 32, 8, "bfloat16", 128, False, 1, True, True, 1.0, 333), (128, 16, 16, "float32", 96, True, 3, True, True, 1.0, 65),
    (128, 5, 5, "float16", 32, False, 2, True, False, 1.25, 3), (64, 1, 1, "float32", 8, True, 1, False, False, 0.75, 2),
    (64, 12, 1, "bfloat16", 48, False, 4, True, True, 1.0, 129), (128, 64, 8, "float16", 64, True, 1, False, False, 1.0, 20),
    (64, 8, 2, "float16", 0, False, 1, True, True, 1.0, 31), (128, 40, 8, "float32", 0, True, 1, False, False, 1.0, 5),
    (64, 8, 2, "bfloat16", 64, False, 2, True, True, 1.0, 601), (128, 4, 1, "float32", 128, True, 1, True, False, 1.0, 1027), (64, 3, 1, "float16", 24, False, 1, False, False, 1.0, 777),
    (128, 2, 1, "bfloat16", 120, False, 3, True, True, 1.0, 17), (64, 33, 11, "float16", 56, False, 1, True, True, 1.0, 9)]


@pytest.mark.parametrize("d,Hq,Hkv,kind,R,neighbours,axes,norm,weights,scale,n", CASES)
def test_against_the_formulas_in_64_bits(d, Hq, Hkv, kind, R, neighbours, axes, norm, weights, scale, n):
    """Projections side by side in one buffer with more columns than heads; positions near and far; each output alone as well."""
    import torch
    t = getattr(torch, kind)
    gen = torch.Generator().manual_seed(d + Hq + R + n)
    wide = (Hq + 2 * Hkv) * d + 32
    x = (torch.randn(n, wide, generator=gen) * torch.exp(torch.randn(n, 1, generator=gen))).to(t)
    x[:, -32:] = float("nan")
    pos = torch.randint(0, 1 << 20, (axes, n), generator=gen, dtype=torch.int32)
    pos[0, :n // 2] = torch.arange(n // 2)
    axis = torch.randint(0, axes, (R // 2,), generator=gen, dtype=torch.uint8)
    w = [(1 + 0.3 * torch.randn(d, generator=gen)).to(t) if weights else None for _ in "qk"]
    inv = frequencies(R) if R else None
    cu = lambda v: None if v is None else v.cuda()
    cfg = sa.make_config(d, Hq, Hkv, sa.SA_KV_FP4)
    rot = sa.Rotary(cfg, cu(torch.from_numpy(inv)) if R else None, dtype=t, pairs="neighbours" if neighbours else "halves", n_axes=axes,
                    pair_axis=cu(axis) if axes > 1 else None, norm=norm, eps=1e-5, scale=scale, q_weight=cu(w[0]), k_weight=cu(w[1]))
    X = x.cuda()
    parts = [v.unflatten(1, (-1, d)) for v in X[:, :-32].split([Hq * d, Hkv * d, Hkv * d], 1)]
    P = pos.cuda() if R else None
    outs = [torch.full((n + 1, h, d), 777.0, dtype=torch.float16, device="cuda") for h in (Hq, Hkv, Hkv)]
    sa.rotate_qkv(rot, *parts, P, *[o[:n] for o in outs])
    alone = [torch.full((n, h, d), 777.0, dtype=torch.float16, device="cuda") for h in (Hq, Hkv, Hkv)]
    for i in range(3):
        sa.rotate_qkv(rot, *[parts[k] if k == i else None for k in range(3)], P, *[alone[k] if k == i else None for k in range(3)])
    torch.cuda.synchronize()
    x64 = x.double().numpy()
    at = [0, Hq * d, (Hq + Hkv) * d, (Hq + 2 * Hkv) * d]
    for i in range(3):
        assert torch.equal(alone[i], outs[i][:n]) and bool((outs[i][n] == 777).all())
        part = x64[:, at[i]:at[i + 1]].reshape(n, -1, d)
        if i < 2:
            y, size = reference(part, R, neighbours, pos.numpy(), axis.long().numpy() * (axes > 1), inv, norm, 1e-5, None if w[i] is None else w[i].double().numpy(), scale)
        else:
            y, size = part, 0.0 * part
        got = outs[i][:n].double().cpu().numpy()
        assert (np.abs(got - y) <= tolerance(y, size)).all(), (i, np.max(np.abs(got - y) / tolerance(y, size)))


def test_far_and_negative_positions():
    """Angles of positions up to 2^30 and below 0: the fraction of a turn is taken in 64 bits."""
    import torch
    d, n = 128, 40
    pos = np.concatenate([2 ** np.arange(30), -(2 ** np.arange(10))]).astype(np.int32)
    x = np.random.default_rng(1).standard_normal((n, 2, d)).astype(np.float32)
    inv = frequencies(d, 5e5)
    cfg = sa.make_config(d, 2, 1, sa.SA_POTM4)
    rot = sa.Rotary(cfg, torch.from_numpy(inv).cuda(), dtype=torch.float32)
    out = torch.zeros(n, 2, d, dtype=torch.float16, device="cuda")
    sa.rotate_qkv(rot, torch.from_numpy(x).cuda(), None, None, torch.from_numpy(pos).cuda(), out, None, None)
    y, size = reference(x.astype(np.float64), d, False, pos[None], np.zeros(d // 2, int), inv, False, 0.0, None, 1.0)
    # (a product of 55 bits in 53: at 2^30 radians 2^-24 of a radian)
    assert (np.abs(out.double().cpu().numpy() - y) <= tolerance(y, size) + 2.0 ** -23 * size).all()


def test_in_place_empty_and_extreme_inputs():
    import torch
    d = 64
    cfg = sa.make_config(d, 4, 2, sa.SA_POTM4)
    inv = torch.from_numpy(frequencies(d)).cuda()
    rot = sa.Rotary(cfg, inv, dtype=torch.float16, norm=True, eps=0.0)
    Q = torch.randn(5, 4, d, device="cuda").half()
    Q[1, 2] = 0                                                   # 0 / 0
    Q[2, 0] = 6e4                                                 # squares beyond binary16
    Q[3, 1] = 6e-8
    pos = torch.arange(5, dtype=torch.int32, device="cuda")
    want = torch.zeros_like(Q)
    sa.rotate_qkv(rot, Q, None, None, pos, want, None, None)
    sa.rotate_qkv(rot, Q, None, None, pos, Q, None, None)
    assert torch.equal(Q[want.isfinite()], want[want.isfinite()])
    bad = torch.zeros(5, 4, d, dtype=torch.bool, device="cuda")
    bad[1, 2] = True
    assert torch.equal(want.isnan(), bad) and torch.equal(Q.isnan(), bad) and bool((want[2, 0].float().abs() < 1.5).all())
    none = torch.zeros(0, 4, d, dtype=torch.float16, device="cuda")
    sa.rotate_qkv(rot, none, None, None, pos[:0], none, None, None)
    V = torch.tensor([1e5, -1e5, 65519.0, 1e-9] * 32, device="cuda").reshape(1, 2, d)
    out = torch.zeros(1, 2, d, dtype=torch.float16, device="cuda")
    sa.rotate_qkv(sa.Rotary(cfg, dtype=torch.float32), None, None, V, None, None, None, out)
    assert torch.equal(out, V.half())


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("d,n,extra", [(64, 5, 0), (64, 700, 4), (128, 700, 0), (128, 3, 4)])
def test_rows_that_start_between_32_byte_places(d, n, extra, neighbours):
    """FP32 projections on 16-byte boundaries only, by their address or by their stride: the same bits as from aligned ones."""
    import torch
    cfg, wide = sa.make_config(d, 4, 2, sa.SA_POTM4), 8 * d + extra
    torch.manual_seed(d + n)
    x = torch.randn(n, 8 * d, device="cuda")
    rot = sa.Rotary(cfg, torch.from_numpy(frequencies(d)).cuda(), dtype=torch.float32, pairs="neighbours" if neighbours else "halves", norm=True, eps=1e-6)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    got = []
    for first in (0, 4):
        room = torch.empty(n * wide + 8, device="cuda")[first:first + n * wide].view(n, wide)[:, :8 * d] if first else x
        room.copy_(x)
        out = [torch.full((n, h, d), 7.0, dtype=torch.float16, device="cuda") for h in (4, 2, 2)]
        q, k, v = (part.unflatten(-1, (-1, d)) for part in room.split([4 * d, 2 * d, 2 * d], -1))
        sa.rotate_qkv(rot, q, k, v, pos, *out)
        got.append(out)
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_rows_beyond_32_bits():
    """Tokens whose places in input and output are beyond 2^31 elements."""
    import torch
    n, cfg = (1 << 25) + 3, sa.make_config(64, 1, 1, sa.SA_POTM4)
    x = torch.zeros(n, 1, 64, dtype=torch.bfloat16, device="cuda")
    x[-3:] = torch.randn(3, 1, 64, device="cuda")
    rot = sa.Rotary(cfg, torch.from_numpy(frequencies(64)).cuda(), dtype=torch.bfloat16)
    pos, out = torch.arange(n, dtype=torch.int32, device="cuda"), torch.full((n, 1, 64), 3.0, dtype=torch.float16, device="cuda")
    sa.rotate_qkv(rot, x, None, None, pos, out, None, None)
    y, size = reference(x[-3:].double().cpu().numpy(), 64, False, pos[-3:].cpu().numpy()[None], np.zeros(32, int), frequencies(64), False, 0.0, None, 1.0)
    assert (np.abs(out[-3:].double().cpu().numpy() - y) <= tolerance(y, size)).all() and not out[:-3].any()
    del x, out, pos
    torch.cuda.empty_cache()


def test_the_binding_refuses_what_does_not_fit():
    import torch
    d, cfg = 64, sa.make_config(64, 4, 2, sa.SA_KV_FP4)
    inv = torch.from_numpy(frequencies(d)).cuda()
    rot = sa.Rotary(cfg, inv, dtype=torch.float16)
    Q, K = (torch.zeros(6, h, d, dtype=torch.float16, device="cuda") for h in (4, 2))
    pos = torch.arange(6, dtype=torch.int32, device="cuda")
    ok = dict(Q=Q, K=K, V=K, positions=pos, Q_out=Q.clone(), K_out=K.clone(), V_out=K.clone())
    sa.rotate_qkv(rot, **ok)
    for name, bad in (("Q", Q.float()), ("Q", Q.cpu()), ("Q", K), ("K", K[:5]), ("V", torch.zeros(6, 2, 2 * d, dtype=torch.float16, device="cuda")[..., ::2]),
                      ("positions", pos.long()), ("positions", pos[:5]), ("positions", pos[None].repeat(2, 1)), ("positions", pos.cpu()),
                      ("Q_out", Q.float()), ("K_out", K[:5]), ("V_out", torch.zeros(12, 2, d, dtype=torch.float16, device="cuda")[::2]), ("Q_out", Q.cpu())):
        with pytest.raises(ValueError):
            sa.rotate_qkv(rot, **{**ok, name: bad})
    for name in ("Q", "Q_out", "positions"):
        with pytest.raises(sa.SaError) as err:
            sa.rotate_qkv(rot, **{**ok, name: None})
        assert err.value.status == 1
    with pytest.raises(sa.SaError) as err:                        # an address between two 16-byte places
        odd = torch.zeros(6 * 4 * d + 8, dtype=torch.float16, device="cuda")[4:-4].view(6, 4, d)
        sa.rotate_qkv(rot, **{**ok, "Q": odd})
    assert err.value.status == 3
    for bad in (dict(inv_freq=inv.double()), dict(inv_freq=inv[::2]), dict(inv_freq=inv, q_weight=torch.ones(d, device="cuda")),
                dict(inv_freq=inv, pair_axis=torch.zeros(3, dtype=torch.uint8, device="cuda")), dict(inv_freq=inv.cpu()), dict(inv_freq=inv, pairs="thirds")):
        with pytest.raises(ValueError):
            sa.Rotary(cfg, **{"dtype": torch.float16, **bad})
    with pytest.raises(ValueError):
        sa.Rotary(cfg, inv, dtype=torch.int16)


@pytest.mark.parametrize("code", [sa.SA_KV_FP4, sa.SA_POTM4])
def test_a_prompt_and_steps_from_projections_to_outputs(code):
    """As a serving loop has it: a prompt's projections are normed, rotated and put into the cache, then tokens are decoded, the step captured
    once and replayed with new projections and positions; the outputs against 64 bits, and the cache read back at the end."""
    import torch
    d, Hq, Hkv, B, n = 64, 8, 2, 3, 4
    lens = np.array([70, 5, 0])
    gen = torch.Generator().manual_seed(code)
    wide = (Hq + 2 * Hkv) * d
    w = [(1 + 0.2 * torch.randn(d, generator=gen)).bfloat16() for _ in "qk"]
    inv = frequencies(d)
    cfg = sa.make_config(d, Hq, Hkv, code)
    rot = sa.Rotary(cfg, torch.from_numpy(inv).cuda(), dtype=torch.bfloat16, norm=True, q_weight=w[0].cuda(), k_weight=w[1].cuda())
    cache = sa.PagedCache(cfg, lens, "cuda", extra_tokens=n)
    split = lambda x: [v.unflatten(1, (-1, d)) for v in x.split([Hq * d, Hkv * d, Hkv * d], 1)]
    rows = lambda k: [torch.zeros(k, h, d, dtype=torch.float16, device="cuda") for h in (Hq, Hkv, Hkv)]
    prompt = torch.randn(int(lens.sum()), wide, generator=gen).bfloat16()
    cu = np.concatenate([[0], np.cumsum(lens)])
    Qp, Kp, Vp = rows(len(prompt))
    where = np.concatenate([np.arange(k) for k in lens]).astype(np.int32)
    sa.rotate_qkv(rot, *split(prompt.cuda()), torch.from_numpy(where).cuda(), Qp, Kp, Vp)
    cache.fill(Kp, Vp, cu)
    x, pos = torch.zeros(B, wide, dtype=torch.bfloat16, device="cuda"), cache.seq_lens.clone()
    Q, K, V = rows(B)
    O = torch.full((B, Hq, d), float("nan"), device="cuda")

    def step():
        pos.copy_(cache.seq_lens)
        sa.rotate_qkv(rot, *split(x), pos, Q, K, V)
        sa.decode_step(cfg, cache.handle, Q, K, V, O, cache.workspace)

    new, outs, seen = [torch.randn(B, wide, generator=gen).bfloat16() for _ in range(n)], [], []
    graph = None
    for i in range(n):
        x.copy_(new[i])
        if i == 1:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        graph.replay() if graph else step()
        torch.cuda.synchronize()
        outs.append(O.cpu().numpy().copy())
        seen.append([v.cpu().numpy().copy() for v in (Q, K, V)])
    total = lens + n
    cu2 = np.concatenate([[0], np.cumsum(total)])
    Kr, Vr = (torch.zeros(int(cu2[-1]), Hkv, d, dtype=torch.float16, device="cuda") for _ in "kv")
    sa.read_kv(cfg, cache.handle, None, cu2, Kr, Vr)
    Kr, Vr, Kp, Vp = (v.cpu().numpy() for v in (Kr, Vr, Kp, Vp))
    for b in range(B):
        for i in range(n):
            # the rows that came out of the rotation, against the formulas
            part = new[i][b].double().numpy()
            for k, (lo, h) in enumerate(((0, Hq), (Hq * d, Hkv))):
                y, size = reference(part[lo:lo + h * d].reshape(1, h, d), d, False, np.array([[lens[b] + i]]), np.zeros(d // 2, int), inv, True, 1e-6,
                                    w[k].double().numpy(), 1.0)
                assert (np.abs(seen[i][k][b] - y[0]) <= tolerance(y, size)[0]).all()
            # attention over what the cache holds
            held = slice(int(cu2[b]), int(cu2[b]) + int(lens[b]) + i + 1)
            ref, against = fp4.attention(seen[i][0][b:b + 1], Kr[held], Vr[held], np.array([0, lens[b] + i + 1]), Hq // Hkv)
            if code == sa.SA_KV_FP4:
                assert (np.abs(outs[i][b] - ref[0]) <= fp4.tolerance(against, d, 80)[0]).all()
            else:                                                 # (queries of 8 bits, keys read as binary16: the tolerance of the other parity tests)
                assert np.abs(outs[i][b] - ref[0]).max() <= 0.1
    if code == sa.SA_KV_FP4:
        K = np.concatenate([np.concatenate([Kp[cu[b]:cu[b + 1]]] + [s[1][b:b + 1] for s in seen]) for b in range(B)])
        V = np.concatenate([np.concatenate([Vp[cu[b]:cu[b + 1]]] + [s[2][b:b + 1] for s in seen]) for b in range(B)])
        assert np.array_equal(Kr.astype(np.float64), fp4.quantised(K)) and np.array_equal(Vr.astype(np.float64), fp4.quantised(V))


def test_queries_are_complete_when_a_decode_call_reads_them_early():
    """The decode kernel reads Q before it waits for the kernel in front of it: that one must be done with Q by then, every time."""
    import torch
    d, Hq, Hkv, B = 128, 32, 8, 16
    cfg = sa.make_config(d, Hq, Hkv, sa.SA_KV_FP4)
    case = synth.make_case("early", [300] * B, Hq, Hkv, d, 0, seed=4)
    c = sa.PagedCache(cfg, case.lens, "cuda")
    bits = lambda v: torch.from_numpy(v).cuda()
    c.fill(bits(case.K), bits(case.V), case.cu_lens)
    rot = sa.Rotary(cfg, dtype=torch.float16)
    inputs = [torch.randn(B, Hq, d, device="cuda").half() for _ in range(4)]
    Q, O = torch.zeros(B, Hq, d, dtype=torch.float16, device="cuda"), [torch.zeros(B, Hq, d, device="cuda") for _ in range(100)]
    want = []
    for x in inputs:
        o = torch.zeros(B, Hq, d, device="cuda")
        torch.cuda.synchronize()
        sa.decode_attention(cfg, c.handle, x, o, c.workspace)
        torch.cuda.synchronize()
        want.append(o)
    for i in range(100):
        sa.rotate_qkv(rot, inputs[i % 4], None, None, None, Q, None, None)
        sa.decode_attention(cfg, c.handle, Q, O[i], c.workspace)
    torch.cuda.synchronize()
    assert all(torch.equal(O[i], want[i % 4]) for i in range(100))
