"""The 4-bit cache (SA_KV_FP4): its writing byte for byte, the decode attention, steps and their forms, against the numpy reference."""
import numpy as np
import pytest

import fp4_reference as fp4
from paper_2609_09208_b200 import binding as sa
from paper_2609_09208_b200 import build as sa_build
from paper_2609_09208_b200 import synth
from test_gpu_stream import EDGES, MIX, marks, up, wide_cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    sa_build.build()


def config(d, Hq, Hkv, hadamard=False):
    return sa.make_config(d, Hq, Hkv, sa.SA_KV_FP4, hadamard=hadamard)


def halves(cache, d):
    """The pool as [page, KV head, half, bytes]."""
    return cache.pages.cpu().numpy().reshape(cache.n_pages, -1, 2, 36 * d)


def plus_zero(code):
    return np.where(code & 7, code, 0)


def poisoned(cfg, lens, *, room=0, extra=0, seed=5, fill=0xff):
    """A cache whose pool holds `fill` everywhere (0xff: scales that are NaN)."""
    c = wide_cache(cfg, lens, room, extra, seed) if room else sa.PagedCache(
        cfg, lens, "cuda", extra_tokens=extra, permutation=synth.page_permutation(int(np.maximum((np.asarray(lens) + extra + 63) // 64, 1).sum()), seed))
    c.pages.fill_(fill)
    return c


def check_cache(c, K, V, cu, hadamard, first=None):
    """Every token of every sequence holds the reference's codes and scales; every other byte or nibble is as `first` (the pool before)."""
    d = K.shape[-1]
    pool, table = halves(c, d), c.page_table.cpu().numpy()
    kc, ks = fp4.encode(fp4.hadamard(K) if hadamard else K)
    vc, vs = fp4.encode(V)
    for b in range(len(cu) - 1):
        for t0 in range(0, int(cu[b + 1] - cu[b]), 32):
            n = min(32, int(cu[b + 1] - cu[b]) - t0)
            rows = slice(int(cu[b]) + t0, int(cu[b]) + t0 + n)
            for h in range(pool.shape[1]):
                got = fp4.unpack(pool[table[b, t0 // 64], h, t0 // 32 % 2], d)
                assert np.array_equal(plus_zero(got[0][:n]), kc[rows, h]) and np.array_equal(got[1][:n], ks[rows, h]), ("keys", b, t0, h)
                assert np.array_equal(plus_zero(got[2][:n]), vc[rows, h]) and np.array_equal(got[3][:n], vs[rows, h]), ("values", b, t0, h)
                if first is not None:
                    was = fp4.unpack(first[table[b, t0 // 64], h, t0 // 32 % 2], d)
                    assert all(np.array_equal(x[n:], y[n:]) for x, y in zip(got, was)), ("behind the end", b, t0, h)


@pytest.mark.parametrize("d,Hkv,hadamard,lens", [
    (64, 4, False, [0, 1, 31, 32, 33, 63, 64, 65, 200]), (64, 1, True, [7, 129]), (128, 8, False, [15, 16, 17, 1, 95]), (128, 2, True, [40, 64, 3]),
    (64, 2, False, [(13 * i) % 90 for i in range(150)])])
def test_fill_byte_for_byte(d, Hkv, hadamard, lens):
    cfg = config(d, Hkv, Hkv, hadamard)
    case = synth.make_case("fp4", lens, Hkv, Hkv, d, 0, outliers=True, seed=d + Hkv)
    case.V[::3] *= np.float16(40.0)
    c = poisoned(cfg, lens, fill=0xa7)
    first = halves(c, d).copy()
    c.fill(up(case.K), up(case.V), case.cu_lens)
    check_cache(c, case.K, case.V, case.cu_lens, hadamard, first)
    used = {int(c.page_table[b, t // 64]) * 2 + t // 32 % 2 for b, n in enumerate(lens) for t in range(0, n, 32)}
    left = [i for i in range(2 * c.n_pages) if i not in used]
    assert np.array_equal(halves(c, d).transpose(0, 2, 1, 3).reshape(2 * c.n_pages, -1)[left], first.transpose(0, 2, 1, 3).reshape(2 * c.n_pages, -1)[left])


def test_rounding_of_every_magnitude():
    """Every binary16 number below a block's largest, for scales of every mantissa, subnormal ones and the saturated one."""
    blocks = []
    for amax in [6 * 1.0, 6 * 1.125, 6 * 1.25, 6 * 1.375, 6 * 1.5, 6 * 1.625, 6 * 1.75, 6 * 1.875, 6.2, 1.0, 65504.0, 61440.0, 61400.0, 2.0 ** -14, 5e-4, 1e-4, 3e-5]:
        top = int(np.float16(amax).view(np.uint16))
        x = np.arange(0, top, max(1, top // 8000), dtype=np.uint16)
        x = np.resize(x, (len(x) + 14) // 15 * 15).reshape(-1, 15)
        b = np.concatenate([np.full((len(x), 1), top, np.uint16), x], 1)
        b[:, 1::2] |= 0x8000
        blocks.append(b)
    blocks = np.concatenate(blocks).view(np.float16)
    K = np.resize(blocks, (len(blocks) // 4 * 4, 16)).reshape(-1, 1, 64)
    n = len(K)
    c = poisoned(config(64, 1, 1), [n])
    cu = np.array([0, n])
    c.fill(up(K), up(K[:, :, ::-1]), cu)
    check_cache(c, K, np.ascontiguousarray(K[:, :, ::-1]), cu, False)


@pytest.mark.parametrize("d,Hkv,hadamard", [(64, 4, False), (64, 3, True), (128, 8, False), (128, 1, True)])
def test_append_writes_what_the_fill_writes(d, Hkv, hadamard):
    """Token by token from various lengths: the bytes of a fill, whatever the pool held, and the other nibble of each byte left alone."""
    import torch
    lens, n = np.array([0, 1, 30, 31, 63, 64, 100]), 5
    cfg = config(d, Hkv, Hkv, hadamard)
    full = synth.make_case("fp4a", lens + n, Hkv, Hkv, d, 0, outliers=True, seed=d + 7 * Hkv)
    B = len(lens)
    old = np.concatenate([np.arange(full.cu_lens[b], full.cu_lens[b] + lens[b]) for b in range(B)]).astype(np.int64)
    got, want = (poisoned(cfg, lens, extra=n, fill=0x5a) for _ in range(2))
    first = halves(got, d).copy()
    got.fill(up(full.K[old]), up(full.V[old]), np.concatenate([[0], np.cumsum(lens)]))
    want.fill(up(full.K), up(full.V), full.cu_lens)
    for i in range(n):
        row = full.cu_lens[:-1] + lens + i
        sa.append_kv(cfg, got.handle, up(full.K[row]), up(full.V[row]), i != 2)
        if i == 2:
            assert np.array_equal(got.seq_lens.cpu().numpy(), lens + 2)
            got.seq_lens += 1
    assert torch.equal(got.seq_lens.cpu(), torch.from_numpy((lens + n).astype(np.int32))) and torch.equal(got.pages, want.pages)
    check_cache(got, full.K, full.V, full.cu_lens, hadamard, first)


def attend(cfg, c, Q, O, **more):
    sa.decode_attention(cfg, c.handle, Q, O, c.workspace, **more)


def run(d, Hq, Hkv, lens, *, hadamard=False, room=0, seed=0, scale=1.0, K=None, V=None):
    import torch
    cfg = config(d, Hq, Hkv, hadamard)
    case = synth.make_case("fp4d", lens, Hq, Hkv, d, 0, outliers=True, seed=1000 + seed)
    K, V = case.K if K is None else K, case.V if V is None else V
    Q = (case.Q.astype(np.float32) * scale).astype(np.float16)
    c = poisoned(cfg, lens, room=room)
    c.fill(up(K), up(V), case.cu_lens)
    O = torch.full((len(lens), Hq, d), float("nan"), device="cuda")
    attend(cfg, c, up(Q), O)
    torch.cuda.synchronize()
    Kq, Vq = fp4.quantised(fp4.hadamard(K) if hadamard else K), fp4.quantised(V)
    ref, against = fp4.attention(fp4.hadamard(Q) if hadamard else Q, Kq, Vq, case.cu_lens, Hq // Hkv)
    return O.cpu().numpy(), ref, fp4.tolerance(against, d, max(lens)), c


SHAPES = [(64, 32, 4, [1024], False), (64, 1, 1, [1], False), (64, 32, 4, EDGES, True), (64, 6, 2, [95, 1, 0, 700], False), (64, 12, 1, [333], False),
          (64, 16, 1, [64, 63, 1000], True), (64, 5, 5, [129] * 3, False), (128, 32, 8, EDGES + [5000], False), (128, 1, 1, [4097], True),
          (128, 16, 16, [31, 257], False), (128, 40, 8, [2000, 17], False), (128, 7, 1, [700, 64, 3], False), (64, 24, 2, [300, 65], True), (64, 11, 1, [200], False), (64, 32, 4, [20000], False), (64, 8, 2, [(37 * i) % 400 for i in range(130)], False)]


@pytest.mark.parametrize("d,Hq,Hkv,lens,hadamard", SHAPES)
def test_decode_against_64_bits(d, Hq, Hkv, lens, hadamard):
    O, ref, tol, _ = run(d, Hq, Hkv, lens, hadamard=hadamard, seed=len(lens))
    assert np.isfinite(O).all() and (np.abs(O - ref) <= tol).all(), np.max(np.abs(O - ref) / tol)
    for b, n in enumerate(lens):
        assert n or not O[b].any()


STREAM = [(64, 32, 4, MIX, 16384, False), (64, 32, 4, [777] * 30 + [9000] * 7, 16384, False), (64, 32, 4, [95] * 125 + [2000] * 3, 16384, True), (64, 16, 1, MIX * 2, 16384, True),
          (64, 8, 1, [(37 * i) % 400 for i in range(128)], 16384, False), (128, 32, 8, MIX, 16384, False), (128, 16, 16, MIX[:12], 16384, True),
          (64, 5, 5, MIX * 2, 16384, False), (128, 64, 8, MIX, 16384, False)]


@pytest.mark.parametrize("d,Hq,Hkv,lens,room,hadamard", STREAM)
def test_one_block_per_sm_against_64_bits(d, Hq, Hkv, lens, room, hadamard):
    O, ref, tol, c = run(d, Hq, Hkv, lens, room=room, hadamard=hadamard, seed=room + d)
    assert marks(c.workspace) > 1                                  # (its counting words: the call went to that kernel)
    assert np.isfinite(O).all() and (np.abs(O - ref) <= tol).all(), np.max(np.abs(O - ref) / tol)


@pytest.mark.parametrize("B,T,d,Hq,Hkv", [(16, 16384, 64, 32, 4), (4, 20000, 128, 32, 8)])
def test_long_sequences_lose_nothing(B, T, d, Hq, Hkv):
    """Root mean square error of long calls against 64 bits (sampled rows): that of sums rounded at random, far below one that grows with
    the length.  A sum of T / 16 products, each rounded by 2^-24 of itself at most, is off by sqrt(T / 16) 2^-24 of the sums of magnitudes where roundings are random;
    these are sqrt(T) times the mean of T independent values of random sign: T / 4 * 2^-24 of the result, with a cut instead of a rounding twice that."""
    O, ref, tol, _ = run(d, Hq, Hkv, [T] * B, seed=T) if B * T < 100000 else sampled(d, Hq, Hkv, B, T)
    err = np.sqrt(((O - ref) ** 2).mean() / (ref ** 2).mean())
    assert err <= T / 2 * 2.0 ** -24, err
    assert (np.abs(O - ref) <= tol).all()


def sampled(d, Hq, Hkv, B, T):
    import torch
    cfg = config(d, Hq, Hkv)
    case = synth.make_case("fp4l", [T] * B, Hq, Hkv, d, 0, outliers=True, seed=3)
    c = sa.PagedCache(cfg, [T] * B, "cuda")
    c.fill(up(case.K), up(case.V), case.cu_lens)
    O = torch.full((B, Hq, d), float("nan"), device="cuda")
    attend(cfg, c, up(case.Q), O)
    pick = [0, B - 1]
    rows = np.concatenate([np.arange(b * T, b * T + T) for b in pick])
    ref, against = fp4.attention(case.Q[pick], fp4.quantised(case.K[rows]), fp4.quantised(case.V[rows]), np.array([0, T, 2 * T]), Hq // Hkv)
    return O[pick].cpu().numpy(), ref, fp4.tolerance(against, d, T), c


@pytest.mark.parametrize("scale", [1e-4, 50.0, 2000.0])
def test_logits_of_every_size(scale):
    """Flat weights, one key that takes all, logits far beyond the exponent's range."""
    O, ref, tol, _ = run(64, 8, 2, [500, 1, 64], scale=scale, seed=5)
    assert np.isfinite(O).all() and (np.abs(O - ref) <= tol).all(), np.max(np.abs(O - ref) / tol)


@pytest.mark.parametrize("d", [64, 128])
def test_extreme_keys_and_values(d):
    """The largest and smallest numbers, blocks of zeros, a block far above its neighbours."""
    lens, H = [300, 40], 2
    rng = np.random.default_rng(2)
    K = (rng.standard_normal((340, H, d)) * 10.0 ** rng.uniform(-6, 0.5, (340, H, d // 16)).repeat(16, -1)).astype(np.float16)
    V = (rng.standard_normal((340, H, d)) * 10.0 ** rng.uniform(-7, 4.2, (340, H, d // 16)).repeat(16, -1)).astype(np.float16)
    V[5], V[6], K[7], V[8, :, 16:32] = 65504, -65504, 0, 0
    O, ref, tol, _ = run(d, 8, H, lens, K=K, V=V)
    assert np.isfinite(O).all() and (np.abs(O - ref) <= tol).all(), np.max(np.abs(O - ref) / tol)


def test_unmapped_pages_are_skipped():
    import torch
    cfg, lens = config(64, 8, 2), [500, 200]
    case = synth.make_case("fp4u", lens, 8, 2, 64, 0, seed=77)
    c = poisoned(cfg, lens)
    c.fill(up(case.K), up(case.V), case.cu_lens)
    c.page_table[0, 3] = -1
    c.page_table[1, 1] = 1 << 30
    O = torch.full((2, 8, 64), float("nan"), device="cuda")
    attend(cfg, c, up(case.Q), O)
    keep = np.ones(700, bool)
    keep[192:256] = keep[500 + 64:500 + 128] = False
    ref, against = fp4.attention(case.Q, fp4.quantised(case.K[keep]), fp4.quantised(case.V[keep]), np.array([0, 436, 572]), 4)
    assert (np.abs(O.cpu().numpy() - ref) <= fp4.tolerance(against, 64, 500)).all()


FORMS = [(64, 32, 4, [0, 1, 31, 63, 64, 500], 0), (64, 5, 1, [40, 200], 0), (128, 28, 4, [900, 0, 64], 0), (64, 12, 2, MIX, 16384), (64, 32, 4, [95] * 125 + [2000] * 3, 2048), (64, 8, 1, [2047], 0), (64, 32, 2, [33, 100], 0), (128, 32, 8, [0, 15, 128, 700], 0),
         (128, 16, 16, [62, 63], 0), (64, 32, 4, MIX, 16384), (128, 32, 8, MIX, 16384), (64, 4, 4, [(7 * i) % 62 for i in range(130)], 0)]


@pytest.mark.parametrize("hadamard", [False, True])
@pytest.mark.parametrize("d,Hq,Hkv,lens,room", FORMS)
def test_steps_equal_append_and_decode(d, Hq, Hkv, lens, room, hadamard):
    """Steps from device and from host buffers, as calls and replayed from a graph: bytes, lengths and outputs of append and decode."""
    import torch
    lens, n, B = np.asarray(lens), 3, len(lens)
    full = synth.make_case("fp4s", lens + n, Hq, Hkv, d, 0, outliers=True, seed=d + B + room)
    cfg = config(d, Hq, Hkv, hadamard)
    old = np.concatenate([np.arange(full.cu_lens[b], full.cu_lens[b] + lens[b]) for b in range(B)]).astype(np.int64)
    caches = [poisoned(cfg, lens, room=room, extra=n) for _ in range(3)]
    for c in caches:
        c.fill(up(full.K[old]), up(full.V[old]), np.concatenate([[0], np.cumsum(lens)]))
    ref, step, host = caches
    lens0 = ref.seq_lens.clone()
    new = [full.cu_lens[:-1] + lens + i for i in range(n)]
    Q, K, V = up(full.Q), [up(full.K[x]) for x in new], [up(full.V[x]) for x in new]
    pin = lambda x: x.cpu().pin_memory()
    Qh, Kh, Vh = pin(Q), [pin(x) for x in K], [pin(x) for x in V]
    staging = torch.full((sa.staging_bytes(cfg, B),), 255, dtype=torch.uint8, device="cuda")
    O = [[torch.full((B, Hq, d), float("nan"), device="cuda") for _ in range(n)] for _ in range(2)]
    Oh = [pin(o) for o in O[0]]
    for i in range(n):
        sa.append_kv(cfg, ref.handle, K[i], V[i], True)
        attend(cfg, ref, Q, O[0][i])
    check_cache(ref, full.K, full.V, full.cu_lens, hadamard)

    def steps():
        for i in range(n):
            sa.decode_step(cfg, step.handle, Q, K[i], V[i], O[1][i], step.workspace)
            sa.decode_step_host(cfg, host.handle, Qh, Kh[i], Vh[i], Oh[i], staging, host.workspace)

    steps()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.seq_lens.copy_(lens0)
        host.seq_lens.copy_(lens0)
        steps()
    for replay in range(3):
        for c in (step, host):
            assert torch.equal(c.pages, ref.pages) and torch.equal(c.seq_lens, lens0 + n)
        for i in range(n):
            assert torch.equal(O[1][i], O[0][i]) and torch.equal(Oh[i], O[0][i].cpu())
            O[1][i].fill_(float("nan"))
            Oh[i].fill_(float("nan"))
        if replay < 2:
            graph.replay()
            torch.cuda.synchronize()


def test_static_scratch_stages_and_repeats_give_the_same_bits():
    import torch
    cfg, lens = config(64, 32, 4), [5000, 0, 333, 64]
    case = synth.make_case("fp4r", lens, 32, 4, 64, 0, seed=12)
    c = poisoned(cfg, lens)
    c.fill(up(case.K), up(case.V), case.cu_lens)
    Q, O = up(case.Q), [torch.full((4, 32, 64), float("nan"), device="cuda") for _ in range(4)]
    attend(cfg, c, Q, O[0])
    sa.decode_attention_static(cfg, c.handle, Q, O[1])
    attend(cfg, c, Q, O[2], stages=1)
    attend(cfg, c, Q, O[2], stages=2)
    c.workspace.fill_(255)
    attend(cfg, c, Q, O[3])
    torch.cuda.synchronize()
    assert torch.equal(O[0], O[1]) and torch.equal(O[0], O[3]) and not O[0][1].any()
    # (in stages the merge kernel may add the same partials, at most 8 here, in another order than the blocks themselves: 7 roundings of 2^-24 each in the sums of
    # either, two for the quotient, on both sides)
    _, (_, size, _) = fp4.attention(case.Q, fp4.quantised(case.K), fp4.quantised(case.V), case.cu_lens, 8)
    assert (np.abs((O[0] - O[2]).cpu().numpy()) <= 32 * 2.0 ** -24 * size).all()
    with pytest.raises(sa.SaError) as err:
        attend(cfg, c, Q, O[0], dbg_scores=torch.zeros(4 * 32 * 5056, dtype=torch.int32, device="cuda"))
    assert err.value.status == 2


@pytest.mark.parametrize("d,Hq,Hkv,lens,room", [(64, 10, 2, [5000, 333], 0), (128, 14, 2, [20000], 0), (64, 28, 4, MIX, 16384), (128, 40, 8, MIX, 16384), (64, 36, 4, MIX, 16384)])
def test_stages_of_groups_of_any_size(d, Hq, Hkv, lens, room):
    """The decode kernel and the merge of its partials apart, for query groups of 5, 7 and 9 (three heads a block)."""
    import torch
    cfg = config(d, Hq, Hkv)
    case = synth.make_case("fp4g", lens, Hq, Hkv, d, 0, seed=Hq)
    c = poisoned(cfg, lens, room=room)
    c.fill(up(case.K), up(case.V), case.cu_lens)
    Q, O = up(case.Q), [torch.full((len(lens), Hq, d), float("nan"), device="cuda") for _ in range(2)]
    attend(cfg, c, Q, O[0])
    attend(cfg, c, Q, O[1], stages=1)
    attend(cfg, c, Q, O[1], stages=2)
    ref, against = fp4.attention(case.Q, fp4.quantised(case.K), fp4.quantised(case.V), case.cu_lens, Hq // Hkv)
    tol = fp4.tolerance(against, d, max(lens))
    for o in O:
        o = o.cpu().numpy()
        assert np.isfinite(o).all() and (np.abs(o - ref) <= tol).all(), np.max(np.abs(o - ref) / tol)


def test_one_workspace_for_calls_of_different_forms_in_turn():
    """4-bit calls of every form and calls of another code, each after every other on one workspace that starts as 255."""
    import torch
    forms = [(64, 32, 4, sa.SA_KV_FP4, MIX, 16384), (64, 32, 4, sa.SA_KV_FP4, [700, 64, 0, 31], 0), (64, 4, 4, sa.SA_KV_FP4, [33] * 130, 0),
             (128, 32, 8, sa.SA_KV_FP4, [20000], 0), (64, 32, 4, sa.SA_POTM4, MIX, 16384), (128, 32, 8, sa.SA_KV_FP4, MIX, 16384)]
    calls = []
    for d, Hq, Hkv, code, lens, room in forms:
        cfg = sa.make_config(d, Hq, Hkv, code)
        case = synth.make_case("turn", lens, Hq, Hkv, d, 0, seed=d + len(lens))
        c = wide_cache(cfg, lens, room or (max(lens) + 64) // 64 * 64, extra=1)
        c.fill(up(case.K), up(case.V), case.cu_lens)
        new = [up(x[np.minimum(np.arange(len(lens)), len(x) - 1)]) for x in (case.K, case.V)]
        calls.append((cfg, c, up(case.Q), new, c.seq_lens.clone()))

    def run(call, workspace):
        cfg, c, Q, (K, V), lens0 = call
        O = torch.full(Q.shape, float("nan"), device="cuda")
        c.seq_lens.copy_(lens0)
        sa.decode_step(cfg, c.handle, Q, K, V, O, workspace)
        return O, c.seq_lens.clone()

    want = [run(call, call[1].workspace) for call in calls]
    one = torch.full((max(len(call[1].workspace) for call in calls),), 255, dtype=torch.uint8, device="cuda")
    got = [(i, run(calls[i], one)) for a in range(len(calls)) for j in range(len(calls)) for i in (a, j)]
    torch.cuda.synchronize()
    for i, (O, lens) in got:
        assert torch.equal(O, want[i][0]) and torch.equal(lens, calls[i][4] + 1), i


@pytest.mark.parametrize("d,Hq,Hkv,lens,room", [(64, 8, 2, [130, 65, 40], 0), (128, 8, 2, [130, 65, 40], 0), (64, 32, 4, MIX, 16384)])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_infinities_and_nans_show(d, Hq, Hkv, lens, room, bad):
    """In a key: its head's queries of that sequence; in a value: the 16 channels of its block; nothing else.  By fill and by append."""
    import torch
    cfg, B, G = config(d, Hq, Hkv), len(lens), Hq // Hkv
    case = synth.make_case("fp4n", [n + 1 for n in lens], Hq, Hkv, d, 0, seed=31)
    K, V = (torch.from_numpy(x.copy()).view(torch.float16).cuda() for x in (case.K, case.V))
    last = torch.from_numpy(case.cu_lens[1:] - 1).cuda()
    cut = torch.ones(len(K), dtype=torch.bool, device="cuda")
    cut[last] = False
    cu = np.concatenate([[0], np.cumsum(lens)])
    i, j, l = sorted(np.argsort(lens)[-3:])                   # three sequences
    k_at, v_at = int(cu[i] + 7), int(cu[j] + lens[j] - 1)     # by fill: the first one's head 1; the second one's head 0
    Kf, Vf, Kn, Vn = K[cut].clone(), V[cut].clone(), K[last].clone(), V[last].clone()
    Kf[k_at, 1, 33] = bad
    Vf[v_at, 0, 20] = bad
    Vn[l, 1, 5] = bad                                         # by the step: the third one
    Kn[l, 0, d - 1] = bad
    c = wide_cache(cfg, [n + 1 for n in lens], room or 256, extra=1)
    c.fill(Kf, Vf, cu)
    c.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
    O = torch.zeros(B, Hq, d, device="cuda")
    sa.decode_step(cfg, c.handle, up(case.Q), Kn, Vn, O, c.workspace)
    want = torch.zeros(B, Hq, d, dtype=torch.bool)
    want[i, G:2 * G] = True
    want[j, :G, 16:32] = True
    want[l, G:2 * G, :16] = True
    want[l, :G] = True
    assert torch.equal(O.isnan().cpu(), want) and O[~want.cuda()].isfinite().all()
    Kr, Vr = (torch.zeros_like(K) for _ in "kv")
    sa.read_kv(cfg, c.handle, None, case.cu_lens, Kr, Vr)
    wk, wv = (torch.zeros(K.shape, dtype=torch.bool) for _ in "kv")
    seq = case.cu_lens
    wk[seq[i] + 7, 1, 32:48] = True
    wk[seq[l + 1] - 1, 0, d - 16:] = True
    wv[seq[j] + lens[j] - 1, 0, 16:32] = True
    wv[seq[l + 1] - 1, 1, :16] = True
    assert torch.equal(Kr.isnan().cpu(), wk) and torch.equal(Vr.isnan().cpu(), wv)


def test_a_pool_beyond_32_bits():
    """Pages behind the first 4 GB of the pool: fill, append, decode, read."""
    import torch
    cfg, n_pages, T = config(128, 16, 8), 62000, 200
    assert n_pages * 8 * sa.get_layout(cfg).page_bytes > 1 << 32
    case = synth.make_case("fp4big", [T + 1], 16, 8, 128, 0, seed=21)
    pages = torch.zeros(n_pages * 8 * sa.get_layout(cfg).page_bytes, dtype=torch.uint8, device="cuda")
    table = torch.tensor([[n_pages - 1, n_pages - 7, n_pages - 2, 58300]], dtype=torch.int32, device="cuda")
    lens = torch.zeros(1, dtype=torch.int32, device="cuda")
    handle = sa.make_cache(pages, table, lens, n_pages)
    workspace = torch.empty(sa.workspace_bytes(cfg, 1, 4), dtype=torch.uint8, device="cuda")
    sa.fill_kv(cfg, handle, up(case.K[:T]), up(case.V[:T]), np.array([0, T]))
    lens.fill_(T)
    O = torch.full((1, 16, 128), float("nan"), device="cuda")
    sa.decode_step(cfg, handle, up(case.Q), up(case.K[T:]), up(case.V[T:]), O, workspace)
    K, V = (torch.zeros(T + 1, 8, 128, dtype=torch.float16, device="cuda") for _ in "kv")
    sa.read_kv(cfg, handle, None, np.array([0, T + 1]), K, V)
    Kq, Vq = fp4.quantised(case.K), fp4.quantised(case.V)
    assert np.array_equal(K.cpu().numpy(), Kq) and np.array_equal(V.cpu().numpy(), Vq)
    ref, against = fp4.attention(case.Q, Kq, Vq, np.array([0, T + 1]), 2)
    assert (np.abs(O.cpu().numpy() - ref) <= fp4.tolerance(against, 128, T)).all()
    del pages
    torch.cuda.empty_cache()


def test_two_streams_with_workspaces_of_their_own():
    import torch
    cfg, lens = config(128, 32, 8), [700, 3000]
    case = synth.make_case("fp4t", lens, 32, 8, 128, 0, seed=13)
    c = poisoned(cfg, lens)
    c.fill(up(case.K), up(case.V), case.cu_lens)
    Q = up(case.Q)
    want = torch.full((2, 32, 128), float("nan"), device="cuda")
    attend(cfg, c, Q, want)
    torch.cuda.synchronize()
    streams, spaces = [torch.cuda.Stream() for _ in range(2)], [c.workspace, c.workspace.clone()]
    outs = [torch.full((2, 32, 128), float("nan"), device="cuda") for _ in range(8)]
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        with torch.cuda.stream(streams[i % 2]):
            sa.decode_attention(cfg, c.handle, Q, o, spaces[i % 2])
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
