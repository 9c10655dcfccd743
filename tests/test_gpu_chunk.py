"""sa_chunk_attention: chunks of new tokens over caches of every code and container, against 64 bits."""
import numpy as np
import pytest

import chunk_reference as ref
from paper_2609_09208_b200 import binding as sa
from paper_2609_09208_b200 import build as sa_build
from paper_2609_09208_b200 import synth
from test_gpu_read import CODES, stored
from test_gpu_stream import up

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    sa_build.build()


class Call:
    """A cache of sequences of `lens` tokens, of which the last `new` are queries."""

    def __init__(self, code, dense, d, Hq, Hkv, lens, new, *, hadamard=False, seed=0, garbage=0xff):
        import torch
        self.cfg = sa.make_config(d, Hq, Hkv, code, nibble=dense, hadamard=hadamard)
        self.code, self.lens, self.new = code, np.asarray(lens), np.asarray(new)
        self.case = synth.make_case("chunk", lens, Hq, Hkv, d, 0, outliers=True, seed=seed + d + code)
        # keys of a layer's size: scores of a few units (log-normal channels alone give some of 40, where one key takes all)
        self.case.K[:] = (self.case.K * np.float16(0.5)).astype(np.float16)
        self.case.V[::5] *= np.float16(1e-5)
        pages = np.maximum((self.lens + 63) // 64, 1)
        self.cache = sa.PagedCache(self.cfg, lens, "cuda", permutation=synth.page_permutation(int(pages.sum()), 3))
        self.cache.pages.fill_(garbage)
        self.cache.fill(up(self.case.K), up(self.case.V), self.case.cu_lens)
        self.cu = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int64)
        rng = np.random.default_rng(seed)
        self.Q = rng.standard_normal((int(self.cu[-1]), Hq, d)).astype(np.float16)
        self.workspace = torch.full((sa.chunk_workspace_bytes(self.cfg, len(lens), len(self.Q)),), 0x5a, dtype=torch.uint8, device="cuda")

    def __call__(self, window=0, sinks=0, dtype=None, O=None):
        import torch
        O = torch.full(self.Q.shape, 777.0, dtype=dtype or torch.float16, device="cuda") if O is None else O
        self.Qd = up(self.Q)
        sa.chunk_attention(self.cfg, self.cache.handle, self.Qd, O, self.workspace, self.cu, window, sinks)
        return O

    def want(self, window=0, sinks=0, there=None, out_step=2.0 ** -11):
        if not hasattr(self, "held"):
            self.held = stored(self.cfg, self.cache, self.code, self.case.K, self.case.V, self.lens)
        K, V = self.held
        cu, q = self.case.cu_lens, ref.queries(self.cfg, self.Q)
        both = [ref.attend(self.cfg, q[self.cu[b]:self.cu[b + 1]], K[cu[b]:cu[b + 1]], V[cu[b]:cu[b + 1]], int(self.lens[b] - self.new[b]), window, sinks,
                           None if there is None else there[b], out_step) for b in range(len(self.lens))]
        return [np.concatenate(x) for x in zip(*both)]


def check(call, *, out_step=2.0 ** -11, dtype=None, there=None, **window):
    got = call(dtype=dtype, **window).double().cpu().numpy()
    want, off = call.want(out_step=out_step, there=there, **window)
    assert np.isfinite(got).all()
    worst = np.max(np.abs(got - want) - off)
    assert worst <= 0, (worst, np.abs(got - want).max())


@pytest.mark.parametrize("d,Hq,Hkv", [(64, 8, 2), (128, 6, 2)])
@pytest.mark.parametrize("code,dense,hadamard", [(*c, h) for c in CODES for h in (False, True) if c[0] != sa.SA_KV_FP16 or not h])
def test_every_code(code, dense, d, Hq, Hkv, hadamard):
    """Chunks of one token, of a few, and of more than a tile of rows, in one call; with and without a window."""
    call = Call(code, dense, d, Hq, Hkv, [200, 131, 64, 300, 1], [1, 7, 64, 290, 1], hadamard=hadamard, seed=1)
    check(call)
    check(call, window=50, sinks=3)


@pytest.mark.parametrize("code,dense", [(sa.SA_POTM4, False), (sa.SA_KV_FP4, False), (sa.SA_KV_FP16, False)])
@pytest.mark.parametrize("d,Hq,Hkv", [(64, 1, 1), (64, 12, 1), (128, 40, 8), (64, 150, 1), (128, 5, 5)])
def test_groups_of_any_size(code, dense, d, Hq, Hkv):
    check(Call(code, dense, d, Hq, Hkv, [140, 33, 257], [3, 1, 30], seed=2))


@pytest.mark.parametrize("n", [1, 2, 4, 5, 8, 9, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257])
def test_chunks_of_every_size(n):
    """Rows around those of which a tile holds one, two or four copies, and around one and two tiles; keys around the ends of tiles and pages."""
    for T in (n, n + 1, n + 63, n + 128, n + 1000):
        check(Call(sa.SA_INT8, False, 64, 8, 2, [T], [n], seed=n))


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 500), (64, 0), (64, 64), (127, 5), (128, 128), (129, 129), (300, 1), (1000, 4), (5000, 7), (2 ** 31 - 1, 2 ** 31 - 1), (0, 9)])
@pytest.mark.parametrize("new", [(1, 1, 1), (6, 40, 200)])
def test_windows(window, sinks, new):
    """Windows and first tokens around pages, tiles and the lengths; sinks without a window say nothing."""
    check(Call(sa.SA_POTM4, False, 64, 4, 2, [700, 41, 1203], new, seed=5), window=window, sinks=sinks)
    check(Call(sa.SA_KV_FP4, False, 128, 4, 2, [700, 41, 1203], new, seed=5), window=window, sinks=sinks)


@pytest.mark.parametrize("code", [sa.SA_POTM2, sa.SA_KV_FP16])
@pytest.mark.parametrize("n", [1, 40])
def test_long_sequences_are_cut(code, n):
    """Few rows over many keys: a unit is cut across the whole machine; and bfloat16 outputs."""
    import torch
    call = Call(code, False, 64, 8, 2, [20001, 777], [n, 1], seed=7)
    check(call)
    check(call, window=9000, sinks=200)
    check(call, dtype=torch.bfloat16, out_step=2.0 ** -8)


@pytest.mark.parametrize("n", [2, 100])
def test_more_units_than_blocks(n):
    """150 sequences (two launches): units within a block, cut ones, several a block; sequences without new tokens and without any."""
    rng = np.random.default_rng(n)
    lens = rng.integers(0, 400, 150)
    lens[::7] = 0
    new = np.minimum(rng.integers(0, n + 1, 150), lens)
    check(Call(sa.SA_POT4, True, 64, 8, 4, lens, new, seed=8))


@pytest.mark.parametrize("code", [sa.SA_KV_FP4, sa.SA_POTM4, sa.SA_KV_FP16])
@pytest.mark.parametrize("new", [2, 150])
def test_pages_that_are_not_mapped(code, new):
    """Keys of such pages are not seen; queries that see none yield zeros."""
    import torch
    call = Call(code, False, 64, 4, 2, [300, 200], [new, new], seed=9)
    call.want()                                                # (what the codes stand for, read while all is mapped)
    table = call.cache.page_table
    table[0, 1], table[0, 3] = -1, 1 << 20
    table[1, :] = -1
    there = [np.ones(300, bool), np.zeros(200, bool)]
    there[0][64:128] = there[0][192:256] = False
    check(call, there=there)
    there[0][:] = False
    table[0, :] = call.cache.n_pages
    assert not call().any()


@pytest.mark.parametrize("code", [sa.SA_KV_FP4, sa.SA_POTM4, sa.SA_INT8, sa.SA_KV_FP16])
@pytest.mark.parametrize("garbage", [0x00, 0x7c, 0xff])
def test_what_nobody_sees_does_not_matter(code, garbage):
    """Slots behind a sequence's end, and tokens outside every window, hold NaN, infinities or anything: the same outputs, bit for bit."""
    import torch
    lens, new = [131, 1000, 65], [1, 40, 5]
    outs = []
    for g in (0x11, garbage):
        call = Call(code, False, 64, 8, 2, lens, new, seed=10, garbage=g)
        pages = call.cache.pages.view(call.cache.n_pages, -1)
        pages[call.cache.page_table[1, 2:12].long()] = g       # tokens 128 .. 767: below the window of the first of 40, above the first tokens
        outs.append(call(window=150, sinks=100))
    torch.cuda.synchronize()
    assert torch.isfinite(outs[0]).all() and torch.equal(*outs)


def test_lengths_shorter_than_their_chunk():
    """Queries at places below zero see nothing."""
    import torch
    call = Call(sa.SA_POTM4, False, 64, 4, 2, [100, 30], [70, 20], seed=11)
    call.cache.seq_lens[:] = torch.tensor([10, 0], dtype=torch.int32)
    got = call()
    assert not got[:60].any() and not got[70:].any() and got[60:70].any((1, 2)).all()
    call.cache.seq_lens[0] = -5
    assert not call().any()


def test_rows_around_a_call_stay():
    """cu_lens from an odd row; rows ahead of the first sequence and behind the last one."""
    import torch
    call = Call(sa.SA_INT8, False, 128, 4, 4, [300, 90, 150], [130, 3, 0], seed=12)
    want = call()
    call.cu = call.cu + 5
    call.Q = np.concatenate([np.full((5, 4, 128), np.nan, np.float16), call.Q, np.full((2, 4, 128), np.nan, np.float16)])
    got = call()
    torch.cuda.synchronize()
    assert torch.equal(got[5:-2], want) and (got[:5] == 777).all() and (got[-2:] == 777).all()


def test_queries_and_scales_at_their_limits():
    """Queries of zeros, queries and keys of the smallest and largest numbers, values up to the largest."""
    import torch
    for code in (sa.SA_POTM4, sa.SA_INT8, sa.SA_KV_FP4, sa.SA_KV_FP16):
        call = Call(code, False, 64, 4, 2, [260, 150], [20, 50], seed=13)
        call.Q[3] = 0
        call.Q[5] *= np.float16(2.0 ** -14)
        call.Q[6] *= np.float16(200.0)
        c = call.case
        c.K[10:20] = 0
        c.K[30:40] *= np.float16(2.0 ** -13)
        c.K[50] = 600.0
        c.V[100] = np.linspace(-65504, 65504, 64)
        c.V[101] = 2.0 ** -24
        c.V[102] = 0
        call.cache.fill(up(c.K), up(c.V), c.cu_lens)
        got = call().double().cpu().numpy()
        want, off = call.want()
        # values of 2^16 (a half step above the largest) may come out as the largest
        off += np.where(np.abs(want) > 65000, 40.0, 0.0)
        want = np.clip(want, -65504, 65504)
        assert np.isfinite(got).all() and (np.abs(got - want) <= off).all(), code


def test_the_same_call_twice_and_a_captured_one():
    """Bit for bit; a captured call follows the lengths; a workspace shared by calls of other shapes and filled with anything in between."""
    import torch
    call = Call(sa.SA_POTM4, False, 64, 8, 2, [3000, 500, 1200], [1, 30, 4], seed=14)
    one = call()
    other = Call(sa.SA_KV_FP4, False, 128, 4, 4, [900], [300], seed=15)
    if other.workspace.numel() > call.workspace.numel():
        call.workspace = other.workspace
    other.workspace = call.workspace
    other()
    call.workspace.fill_(0xff)
    two = call()
    torch.cuda.synchronize()
    assert torch.equal(one, two)
    O, Q = torch.zeros_like(one), call.Qd                      # (the captured call's own: other calls make their own copy)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sa.chunk_attention(call.cfg, call.cache.handle, Q, O, call.workspace, call.cu)
    for shorter in (0, 17, 400):
        call.cache.seq_lens[:] = torch.tensor([3000 - shorter, 500 - shorter, 1200 - shorter], dtype=torch.int32)
        graph.replay()
        torch.cuda.synchronize()
        got = O.clone()
        assert torch.equal(got, call())
    del graph


def test_two_calls_at_once():
    """On two streams, each with its own workspace."""
    import torch
    calls = [Call(c, False, 64, 8, 2, [4000, 100], [3, 90], seed=16 + i) for i, c in enumerate((sa.SA_POTM4, sa.SA_KV_FP4))]
    want = [c() for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    got = [[], []]
    for _ in range(20):
        for c, s, g in zip(calls, streams, got):
            with torch.cuda.stream(s):
                g.append(torch.zeros_like(want[0]))
                sa.chunk_attention(c.cfg, c.cache.handle, c.Qd, g[-1], c.workspace, c.cu)
    torch.cuda.synchronize()
    assert all(torch.equal(x, w) for w, g in zip(want, got) for x in g)


def test_one_token_is_a_decode_step():
    """A chunk of one token a sequence is what the decode call computes, up to the rounding of weights and outputs."""
    import torch
    for code in (sa.SA_POTM4, sa.SA_POT4, sa.SA_INT8, sa.SA_KV_FP4, sa.SA_KV_FP16):
        call = Call(code, False, 64, 8, 2, [1000, 77, 300], [1, 1, 1], seed=18)
        O = torch.zeros(call.Q.shape, device="cuda")
        got = call().double()
        sa.decode_attention_fp16(call.cfg, call.cache.handle, call.Qd, O, call.cache.workspace) if code == sa.SA_KV_FP16 else \
            sa.decode_attention(call.cfg, call.cache.handle, call.Qd, O, call.cache.workspace)
        off = call.want()[1] + 1e-5
        assert (np.abs((got - O.double()).cpu().numpy()) <= off).all()


def test_a_pool_and_rows_beyond_32_bits():
    """Pages behind the first 2^32 bytes of a pool, and rows of queries and outputs behind the first 2^32 bytes of theirs."""
    import torch
    d, H, n = 128, 8, 90
    small = Call(sa.SA_KV_FP16, False, d, H, H, [300, 130], [n, 1], seed=20)
    want = small(window=200, sinks=10)
    c, page = small.cache, small.cache.layout.page_bytes * H
    far = (1 << 32) // page + 11
    pool = torch.zeros((far + c.n_pages) * page, dtype=torch.uint8, device="cuda")
    pool[far * page:] = c.pages
    table = (c.page_table + far * (c.page_table >= 0)).int()
    handle = sa.make_cache(pool, table, c.seq_lens, far + c.n_pages)
    row0 = (1 << 32) // (2 * d * H) + 3
    Q, O = (torch.zeros(row0 + n + 1, H, d, dtype=torch.float16, device="cuda") for _ in "qo")
    Q[row0:] = small.Qd.view(torch.float16)
    sa.chunk_attention(small.cfg, handle, Q, O, small.workspace, small.cu + row0, 200, 10)
    torch.cuda.synchronize()
    assert torch.equal(O[row0:], want) and not O[:row0].any()


def test_on_another_stream_behind_the_writes():
    """A chain on a side stream: cache written, attended to and written again, over and over; every output is that of its own cache."""
    import torch
    calls = [Call(sa.SA_POTM2, False, 64, 4, 2, [700, 65], [40, 2], seed=21 + i) for i in range(2)]
    want = [c() for c in calls]
    torch.cuda.synchronize()
    one, stream, got = calls[0], torch.cuda.Stream(), []
    rows = [(up(c.case.K), up(c.case.V)) for c in calls]
    with torch.cuda.stream(stream):
        for i in range(30):
            sa.fill_kv(one.cfg, one.cache.handle, *rows[i % 2], one.case.cu_lens)
            got.append(torch.zeros_like(want[0]))
            sa.chunk_attention(one.cfg, one.cache.handle, calls[i % 2].Qd, got[-1], one.workspace, one.cu)
    torch.cuda.synchronize()
    assert all(torch.equal(g, want[i % 2]) for i, g in enumerate(got))


@pytest.mark.parametrize("code,dense", [(sa.SA_POTM4, False), (sa.SA_POT4, True), (sa.SA_KV_FP16, False), (sa.SA_KV_FP4, False)])
@pytest.mark.parametrize("d", [64, 128])
def test_the_same_outputs_over_and_over(code, dense, d):
    """Calls of every kind of row tile, fifty times: bit for bit (a wait that is missing shows here)."""
    import torch
    for lens, new in (([5000, 3000, 900], [1, 4, 3]), ([5000, 3000, 900], [8, 5, 8]), ([5000, 3000], [13, 16]), ([3000, 1500], [200, 700])):
        call = Call(code, dense, d, 8, 2, lens, new, seed=23)
        first = call()
        others = [call() for _ in range(50)]
        torch.cuda.synchronize()
        assert all(torch.equal(first, o) for o in others)


@pytest.mark.parametrize("d,Hq,Hkv", [(64, 8, 2), (128, 6, 2)])
@pytest.mark.parametrize("code", [sa.SA_POTM4, sa.SA_POT4, sa.SA_INT8, sa.SA_KV_FP4, sa.SA_KV_FP16])
@pytest.mark.parametrize("new", [(5, 5), (90, 90), (9, 300)])
def test_queries_that_are_no_numbers(code, d, Hq, Hkv, new):
    """A query with an infinity or a NaN yields NaN, also where all its scores are minus infinity; zeros where it sees no token; and no other row changes."""
    import torch
    call = Call(code, False, d, Hq, Hkv, [310, 305], new, seed=24)
    K = call.case.K
    K[..., 3] = np.abs(K[..., 3]) + np.float16(0.5)            # a channel that no key has negative or zero
    call.cache.fill(up(K), up(call.case.V), call.case.cu_lens)
    call.cache.seq_lens[0] = new[0] - 3                        # its first three queries see nothing, the fourth one token
    clean = call()
    rng = np.random.default_rng(3)
    bad = np.zeros(call.Q.shape[:2], bool)
    for row in (0, 1, 2, 3, 4, new[0] - 1, new[0], new[0] + 1, new[0] + 3, len(call.Q) - 1):
        for h, x in zip(rng.permutation(Hq)[:3], (np.nan, np.inf, -np.inf)):
            call.Q[row, h, 3] = x
            bad[row, h] = True
    got = call()
    torch.cuda.synchronize()
    bad = torch.from_numpy(bad).cuda()
    nothing = torch.zeros_like(bad)
    nothing[:3] = True
    assert torch.equal(got[~bad], clean[~bad]) and not got[nothing].any() and not clean[nothing].any()
    assert got[bad & ~nothing].isnan().all()


@pytest.mark.parametrize("d,Hq,Hkv", [(64, 8, 2), (128, 6, 2)])
@pytest.mark.parametrize("code", [sa.SA_POTM4, sa.SA_POT4, sa.SA_INT8, sa.SA_KV_FP4, sa.SA_KV_FP16])
@pytest.mark.parametrize("new", [1, 40, 200])
def test_tokens_that_are_no_numbers(code, d, Hq, Hkv, new):
    """A key with a NaN shows in every query that sees it, and in no other sequence or KV head; a value with one too, where the cache can hold it."""
    import torch
    call = Call(code, False, d, Hq, Hkv, [300, 305, 260], [new] * 3, seed=30)
    clean = call()
    cu, c, G = call.case.cu_lens, call.case, Hq // Hkv
    place = 300 - 1 - new // 2                                  # the token of query new - 1 - new // 2
    which = [c.K] + [c.V] * (code in (sa.SA_KV_FP16, sa.SA_KV_FP4))
    for x in which:
        keep = x[cu[0] + place, 1].copy()
        x[cu[0] + place, 1, 7] = np.nan
        call.cache.fill(up(c.K), up(c.V), cu)
        got = call()
        torch.cuda.synchronize()
        x[cu[0] + place, 1] = keep
        sees = torch.zeros(call.Q.shape[:2], dtype=torch.bool, device="cuda")
        sees[new - 1 - new // 2:new, G:2 * G] = True
        shows = got.isnan().any(-1)
        assert shows[sees].all() and not shows[new:].any() and not shows[:, :G].any()
        assert torch.equal(got[new:], clean[new:]) and torch.equal(got[:, :G], clean[:, :G])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,n", [(257, 1), (257, 100), (3000, 200), (20000, 2)])
def test_values_of_the_largest_magnitude(d, T, n):
    """Equal values of the largest magnitude: their mean is that number, however the weights have been rounded, and no infinity.  (All keys but the first weigh a bit more than half a
    step of binary16 above a power of two, which the rounding takes up by 2^-11.)"""
    import torch
    call = Call(sa.SA_KV_FP16, False, d, 4, 2, [T], [n], seed=25)
    # q k / sqrt(d) log2(e) = -1 + log2(1 + 2^-11 + a little)
    want = (np.log2(1 + 2.0 ** -11 * 1.03) - 1) * d ** 0.5 / np.log2(np.e)
    q = np.linspace(1, 2, 1024, endpoint=False).astype(np.float16)
    k = (want / q.astype(np.float64)).astype(np.float16)
    best = np.abs(q.astype(np.float64) * k.astype(np.float64) - want).argmin()
    call.Q[:] = 0
    call.Q[..., 0] = q[best]
    c = call.case
    c.K[:] = 0
    c.K[1:, :, 0] = k[best]
    c.V[:] = 65504
    c.V[..., ::2] = -65504
    call.cache.fill(up(c.K), up(c.V), c.cu_lens)
    for dtype in (torch.float16, torch.bfloat16):
        got = call(dtype=dtype).double()
        torch.cuda.synchronize()
        # (weights off by 2^-11 at most, then the output's rounding)
        assert ((got.abs() - 65504).abs() <= 65504 * (2.0 ** -11 + (0 if dtype == torch.float16 else 2.0 ** -8 * 1.01))).all(), (got.abs().max(), got.abs().min())
        assert (got[..., ::2] < 0).all() and (got[..., 1::2] > 0).all()


@pytest.mark.parametrize("d,code,new", [(64, sa.SA_POTM4, 1), (128, sa.SA_KV_FP4, 3), (64, sa.SA_INT8, 60), (128, sa.SA_KV_FP16, 40)])
@pytest.mark.parametrize("batch", [36, 37])
def test_about_as_many_units_as_blocks(d, code, new, batch):
    """144 and 148 units, equal and ragged: a unit a block, or cut ones; a captured call decides by the lengths that it finds."""
    import torch
    rng = np.random.default_rng(batch)
    lens = rng.integers(new, 300, batch)
    lens[5] = 6000
    call = Call(code, False, d, 16, 4, lens, [new] * batch, seed=26)
    check(call)
    check(call, window=100, sinks=7)
    ragged, equal = call(), torch.full((batch,), int(min(lens)), dtype=torch.int32, device="cuda")
    lengths = call.cache.seq_lens.clone()
    call.cache.seq_lens.copy_(equal)
    short, O, Q = call(), torch.zeros_like(ragged), call.Qd
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sa.chunk_attention(call.cfg, call.cache.handle, Q, O, call.workspace, call.cu)
    for now, want in ((equal, short), (lengths, ragged), (equal, short)):
        call.cache.seq_lens.copy_(now)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(O, want)
    del graph


def test_one_long_sequence_beside_short_ones():
    """148 units of which 4 have 256 tiles of keys and the others one: about as long as the long sequence by itself and the others by themselves, not a block's walk through 256 tiles."""
    import torch

    def time(lens):
        call = Call(sa.SA_POTM4, False, 64, 32, 4, lens, [1] * len(lens), seed=27)
        O = call()
        go = lambda: sa.chunk_attention(call.cfg, call.cache.handle, call.Qd, O, call.workspace, call.cu)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for _ in range(20):
                go()
        start, end = (torch.cuda.Event(enable_timing=True) for _ in "se")
        best = np.inf
        for _ in range(10):
            start.record()
            graph.replay()
            end.record()
            torch.cuda.synchronize()
            best = min(best, start.elapsed_time(end))
        del graph
        return best

    both, long, short = time([32768] + [100] * 36), time([32768]), time([100] * 36)
    assert both <= 2 * (long + short), (both, long, short)      # (5 times as long where nothing is cut)


def lost(call, b, kv_head, tile):
    """The rows that the hook's call leaves, where they are NaN, and what they hold else: all of a row is NaN or none."""
    import torch
    O = torch.full(call.Q.shape, 777.0, dtype=torch.float16, device="cuda")
    sa.debug_chunk_lost_copy(call.cfg, call.cache.handle, call.Qd, O, call.workspace, call.cu, b, kv_head, tile)
    torch.cuda.synchronize()
    nan = O.isnan()
    assert torch.equal(nan.any(-1), nan.all(-1))
    return O, nan.all(-1)


@pytest.mark.parametrize("lens,new,at,alone", [
    ([300, 500, 100], [1, 5, 2], (1, 1, 2), True), ([128, 90], [1, 20], (0, 0, 0), True), ([20000, 700], [3, 1], (0, 0, 100), False), ([3000, 500], [700, 400], (0, 1, 10), False),
    ([3000, 500], [700, 400], (1, 0, 0), False), ([900, 200, 640], [30, 1, 400], (2, 1, 4), False)])
def test_a_copy_that_never_comes(lens, new, at, alone):
    """The rows that need the tile are NaN; the others are what they are otherwise, or NaN too where their block had given up (`alone`: blocks have one unit each); the next call is as any."""
    import torch
    call = Call(sa.SA_POTM4, False, 64, 8, 2, lens, new, seed=28)
    want = call()
    O, nan = lost(call, *at)
    b, kv_head, tile = at
    first = max(128 * tile - (lens[b] - new[b]), 0)
    hit = torch.zeros_like(nan)
    hit[call.cu[b] + first:call.cu[b + 1], 4 * kv_head:4 * kv_head + 4] = True
    assert hit.any() and nan[hit].all() and torch.equal(O[~nan], want[~nan])
    if alone:
        assert torch.equal(nan, hit)
    assert torch.equal(call(), want)


@pytest.mark.parametrize("pieces", [0, 1, 2])
@pytest.mark.parametrize("lens,new", [([20000, 3000], [3, 1]), ([3000, 500], [700, 400]), (range(100, 250), [1] * 150), ([2000] * 20, [60] * 20)])
def test_blocks_that_give_up(lens, new, pieces):
    """Rows that blocks had not handed out yet are NaN, also where an earlier call has left finite sums of theirs in the workspace."""
    import torch
    call = Call(sa.SA_POTM4, False, 64, 8, 2, list(lens), new, seed=29)
    call()
    call.Q[:] = call.Q[::-1].copy()
    workspace, call.workspace = call.workspace, call.workspace.clone()
    want = call()
    call.workspace = workspace
    O, nan = lost(call, 0, 0, -1 - pieces)
    # (a second piece: with 300 units on fewer than 150 blocks some have one, where an equal stretch is shorter than a unit's fixed cost of 4 tiles and two more none has)
    assert torch.equal(O[~nan], want[~nan]) and (nan.all() if pieces == 0 else nan.any() or pieces == 2 or len(lens) < 150)
    assert torch.equal(call(), want)
