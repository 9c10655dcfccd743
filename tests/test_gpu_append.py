"""sa_append_qkv against sa_rotate_qkv and sa_fill_kv, which it does in one: the same bits in the cache and in the queries."""
import numpy as np
import pytest

from paper_2609_09208_b200 import binding as sa
from paper_2609_09208_b200 import build as sa_build
from paper_2609_09208_b200 import synth
from test_gpu_read import CODES

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    sa_build.build()


def rotary(cfg, dtype, *, rotary_dim=None, norm=True, pairs="halves", axes=1, seed=0):
    import torch
    d = cfg.head_dim
    R = d if rotary_dim is None else rotary_dim
    gen = torch.Generator(device="cuda").manual_seed(seed)
    inv = (1e4 ** (-torch.arange(R // 2, device="cuda", dtype=torch.float64) * 2 / max(R, 1))).float() if R else None
    w = [(1 + 0.2 * torch.randn(d, device="cuda", generator=gen)).to(dtype) if norm else None for _ in "qk"]
    axis = (torch.arange(R // 2, device="cuda") % axes).byte() if axes > 1 and R else None
    return sa.Rotary(cfg, inv, dtype=dtype, norm=norm, pairs=pairs, n_axes=axes, pair_axis=axis, q_weight=w[0], k_weight=w[1])


class Calls:
    """Sequences that hold `before` tokens and get `new` ones: the cache as append_qkv leaves it, and as rotate_qkv and fill_kv build it from all rows."""

    def __init__(self, cfg, rot, dtype, before, new, *, axes=1, seed=0, extra=0):
        import torch
        self.cfg, self.rot = cfg, rot
        self.before, self.new = np.asarray(before), np.asarray(new)
        d, Hq, Hkv = cfg.head_dim, cfg.n_q_heads, cfg.n_kv_heads
        gen = torch.Generator(device="cuda").manual_seed(seed)
        total = self.before + self.new
        self.cu_all = np.concatenate([[0], np.cumsum(total)])
        self.cu = np.concatenate([[0], np.cumsum(self.new)])
        n = int(self.cu_all[-1])
        x = torch.randn(n, (Hq + 2 * Hkv) * d, device="cuda", generator=gen)
        x[::3] *= 1e-3
        self.x = x.to(dtype)
        self.pos = torch.stack([torch.randint(0, 200000, (n,), device="cuda", generator=gen) for _ in range(axes)]).int()
        self.rows = [torch.zeros(n, h, d, dtype=torch.float16, device="cuda") for h in (Hq, Hkv, Hkv)]
        sa.rotate_qkv(rot, *self.parts(self.x), self.pos, *self.rows)
        is_new = np.concatenate([np.arange(t) >= b for t, b in zip(total, self.before)] + [np.zeros(0, bool)])
        self.at = torch.from_numpy(np.flatnonzero(is_new)).cuda()
        old = torch.from_numpy(np.flatnonzero(~is_new)).cuda()
        pages = int(np.maximum((total + extra + 63) // 64, 1).sum())
        self.caches = [sa.PagedCache(cfg, total, "cuda", extra_tokens=extra, permutation=synth.page_permutation(pages, 5)) for _ in range(2)]
        for c in self.caches:
            c.pages.fill_(0xa5)
        self.caches[1].fill(self.rows[1], self.rows[2], self.cu_all)
        cu_old = np.concatenate([[0], np.cumsum(self.before)])
        self.caches[0].fill(self.rows[1][old].contiguous(), self.rows[2][old].contiguous(), cu_old)
        self.x_new, self.pos_new = self.x[self.at].contiguous(), self.pos[:, self.at].contiguous()
        self.Q = torch.full((len(self.at), Hq, d), 777.0, dtype=torch.float16, device="cuda")

    def parts(self, x):
        d, Hq, Hkv = self.cfg.head_dim, self.cfg.n_q_heads, self.cfg.n_kv_heads
        return [v.unflatten(1, (-1, d)) for v in x.split([Hq * d, Hkv * d, Hkv * d], 1)]

    def append(self, **kw):
        sa.append_qkv(self.rot, self.caches[0].handle, *self.parts(self.x_new), self.pos_new, self.cu, self.Q, **kw)

    def check(self):
        import torch
        torch.cuda.synchronize()
        assert torch.equal(self.Q.view(torch.int16), self.rows[0][self.at].view(torch.int16))
        assert torch.equal(self.caches[0].pages, self.caches[1].pages)
        assert torch.equal(self.caches[0].seq_lens, self.caches[1].seq_lens)


BEFORE, NEW = [0, 3, 62, 64, 31, 100, 7, 0], [5, 1, 70, 2, 33, 130, 0, 0]


@pytest.mark.parametrize("d,Hq,Hkv", [(64, 8, 2), (128, 3, 3)])
@pytest.mark.parametrize("code,dense,hadamard", [(*c, h) for c in CODES for h in (False, True) if c[0] != sa.SA_KV_FP16 or not h])
def test_every_code(code, dense, d, Hq, Hkv, hadamard):
    import torch
    cfg = sa.make_config(d, Hq, Hkv, code, nibble=dense, hadamard=hadamard)
    c = Calls(cfg, rotary(cfg, torch.bfloat16), torch.bfloat16, BEFORE, NEW, seed=code)
    c.append()
    c.check()


@pytest.mark.parametrize("before,new", [([0], [1]), ([63], [1]), ([5] * 40, [1] * 40), ([1, 2, 3, 4, 5], [1, 1, 1, 1, 1]), ([9], [1500]), ([33, 0], [700, 900]), (range(200), [1] * 200), ([50] * 700, [1] * 700), ([0, 1, 2, 3] * 30, [2, 3, 4, 5] * 30)])
@pytest.mark.parametrize("code", [sa.SA_KV_FP4, sa.SA_POTM4])
def test_from_one_token_to_long_chunks(code, before, new):
    """A block a token, blocks of several, several launches."""
    import torch
    cfg = sa.make_config(64, 4, 4, code)
    c = Calls(cfg, rotary(cfg, torch.float16), torch.float16, list(before), list(new), seed=3)
    c.append()
    c.check()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kw", [dict(pairs="neighbours"), dict(norm=False), dict(rotary_dim=24), dict(rotary_dim=40, pairs="neighbours", axes=3), dict(axes=4), dict(rotary_dim=0)])
def test_rotations_and_types(d, kw):
    import torch
    for dtype in (torch.float16, torch.bfloat16, torch.float32):
        for code in (sa.SA_POTM1, sa.SA_KV_FP4):
            cfg = sa.make_config(d, 6, 2, code)
            c = Calls(cfg, rotary(cfg, dtype, **kw), dtype, [3, 70], [9, 30], axes=kw.get("axes", 1), seed=4)
            c.append()
            c.check()


def test_many_heads():
    """More keys and values than 48 KB of shared memory hold."""
    import torch
    for d, H in ((64, 100), (128, 120)):
        for new in ([1, 1], [6, 3]):
            cfg = sa.make_config(d, H, H, sa.SA_KV_FP4)
            c = Calls(cfg, rotary(cfg, torch.bfloat16), torch.bfloat16, [5, 66], new, seed=5)
            c.append()
            c.check()


@pytest.mark.parametrize("d,new,heads", [(64, [6, 3], (40, 47, 48, 60, 100, 200)), (64, [1, 1], (100, 191, 192, 193, 200)), (128, [6, 3], (47, 48, 64, 96, 200)), (128, [1, 1], (95, 96, 97, 130, 200))])
def test_more_heads_from_call_to_call(d, new, heads):
    """Keys and values around the 48 KB of shared memory that a block has without asking, up to the most, each count above the last: FP32 and neighbouring pairs, a kernel that no other
    test gives as many heads."""
    import torch
    for H in heads:
        cfg = sa.make_config(d, H, H, sa.SA_KV_FP4)
        c = Calls(cfg, rotary(cfg, torch.float32, pairs="neighbours"), torch.float32, [5, 66], new, seed=H)
        c.append()
        c.check()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("code,dense,hadamard", [(*c, h) for c in CODES for h in (False, True) if c[0] != sa.SA_KV_FP16 or not h])
def test_projections_that_are_no_numbers(code, dense, d, hadamard):
    """Infinities, NaN, numbers beyond binary16 and zeros, with and without norms: the codes and queries of rotate_qkv and fill_kv."""
    import torch
    for norm in (False, True):
        for new in ([1, 1, 1], [9, 70, 33]):
            cfg = sa.make_config(d, 4, 2, code, nibble=dense, hadamard=hadamard)
            rot = rotary(cfg, torch.float32, norm=norm)
            c = Calls(cfg, rot, torch.float32, [5, 61, 0], new, seed=11)
            gen = torch.Generator(device="cuda").manual_seed(12)
            at = torch.rand(c.x_new.shape, device="cuda", generator=gen)
            for i, x in enumerate((torch.inf, -torch.inf, torch.nan, 70000.0, -65520.0, 0.0)):
                c.x_new[(at >= 0.002 * i) & (at < 0.002 * (i + 1))] = x
            c.x_new[-1, -d:], c.x_new[-1, 4 * d:5 * d] = 0, 0
            c.x[c.at] = c.x_new
            sa.rotate_qkv(rot, *c.parts(c.x), c.pos, *c.rows)
            c.caches[1].fill(c.rows[1], c.rows[2], c.cu_all)
            c.append()
            c.check()


@pytest.mark.parametrize("code", [sa.SA_KV_FP4, sa.SA_POTM2])
def test_pages_that_are_not_mapped(code):
    """A sequence of which one page is missing is left as it is, its queries are not; the others get their tokens."""
    import torch
    for new in ([70, 10, 1], [1, 1, 1]):
        cfg = sa.make_config(64, 4, 2, code)
        c = Calls(cfg, rotary(cfg, torch.float16), torch.float16, [64, 20, 63], new, seed=6)
        page = (64 + new[0] - 1) // 64
        for cache in c.caches:
            cache.page_table[0, page] = -1 if code == sa.SA_KV_FP4 else cache.n_pages
        before = c.caches[0].pages.clone()
        c.append()
        torch.cuda.synchronize()
        assert c.caches[0].seq_lens.tolist() == [64, 20 + new[1], 63 + new[2]]
        assert torch.equal(c.Q, c.rows[0][c.at])
        got, want, old = (p.view(c.caches[0].n_pages, -1) for p in (c.caches[0].pages, c.caches[1].pages, before))
        own = c.caches[0].page_table[1:].flatten().long()
        own = own[own >= 0]
        assert torch.equal(got[own], want[own])
        rest = torch.ones(len(got), dtype=torch.bool, device="cuda")
        rest[own] = False
        assert torch.equal(got[rest], old[rest])


def test_no_bump_no_queries_and_other_rows():
    import torch
    cfg = sa.make_config(64, 4, 2, sa.SA_POTM4)
    c = Calls(cfg, rotary(cfg, torch.bfloat16), torch.bfloat16, [10, 100], [20, 3], seed=7)
    sa.append_qkv(c.rot, c.caches[0].handle, None, *c.parts(c.x_new)[1:], c.pos_new, c.cu, None, bump_lens=False)
    torch.cuda.synchronize()
    assert c.caches[0].seq_lens.tolist() == [10, 100] and torch.equal(c.caches[0].pages, c.caches[1].pages)
    # rows around those that cu_lens names
    wide = lambda t, dim: torch.cat([t.narrow(dim, 0, 3), t, t.narrow(dim, 0, 2)], dim)
    x, pos = wide(c.x_new, 0), wide(c.pos_new, 1).contiguous()
    Q = torch.full((len(x), 4, 64), 777.0, dtype=torch.float16, device="cuda")
    sa.append_qkv(c.rot, c.caches[0].handle, *c.parts(x), pos, c.cu + 3, Q)
    torch.cuda.synchronize()
    assert torch.equal(Q[3:-2], c.rows[0][c.at]) and (Q[:3] == 777).all() and (Q[-2:] == 777).all()
    assert c.caches[0].seq_lens.tolist() == [30, 103] and torch.equal(c.caches[0].pages, c.caches[1].pages)


@pytest.mark.parametrize("code", [sa.SA_KV_FP4, sa.SA_POTM1])
def test_a_captured_call_follows_the_lengths(code):
    """Chunks of three tokens and of one, recorded once and replayed five times."""
    import torch
    cfg = sa.make_config(64, 4, 2, code)
    for per in (1, 3):
        before, n = [61, 0], 5 * per
        c = Calls(cfg, rotary(cfg, torch.float16), torch.float16, before, [n, n], seed=8)
        x, pos, Q = torch.zeros(2 * per, c.x.shape[1], dtype=torch.float16, device="cuda"), torch.zeros(1, 2 * per, dtype=torch.int32, device="cuda"), torch.zeros(2 * per, 4, 64, dtype=torch.float16, device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            sa.append_qkv(c.rot, c.caches[0].handle, *c.parts(x), pos, np.array([0, per, 2 * per]), Q)
        for i in range(5):
            rows = torch.cat([torch.arange(per, device="cuda") + i * per + s * n for s in range(2)])
            x.copy_(c.x_new[rows])
            pos.copy_(c.pos_new[:, rows])
            graph.replay()
            c.Q[rows] = Q
        c.check()
        del graph


def test_a_serving_loop():
    """Prompts in chunks, drafts, single tokens, each appended and attended to with a window, against 64 bits over the rows that went in (binary16 cache)."""
    import torch
    import chunk_reference as ref
    d, Hq, Hkv = 64, 8, 2
    cfg = sa.make_config(d, Hq, Hkv, sa.SA_KV_FP16)
    steps = [[100, 0, 37], [60, 1, 0], [1, 1, 1], [4, 130, 5], [1, 1, 1], [0, 300, 1]]
    total = np.sum(steps, 0)
    rot = rotary(cfg, torch.bfloat16)
    cache = sa.PagedCache(cfg, total, "cuda")
    cache.pages.fill_(0xff)
    gen = torch.Generator(device="cuda").manual_seed(9)
    held = [[np.zeros((0, Hkv, d), np.float16)] * 3 for _ in "kv"]
    workspace = torch.empty(sa.chunk_workspace_bytes(cfg, 3, 1000), dtype=torch.uint8, device="cuda")
    lens = np.zeros(3, int)
    for i, new in enumerate(steps):
        new = np.array(new)
        cu, n = np.concatenate([[0], np.cumsum(new)]), int(new.sum())
        x = torch.randn(n, (Hq + 2 * Hkv) * d, device="cuda", generator=gen).bfloat16()
        parts = [v.unflatten(1, (-1, d)) for v in x.split([Hq * d, Hkv * d, Hkv * d], 1)]
        pos = torch.from_numpy(np.concatenate([np.arange(a, a + b) for a, b in zip(lens, new)]).astype(np.int32)).cuda()
        rows = [torch.zeros(n, h, d, dtype=torch.float16, device="cuda") for h in (Hq, Hkv, Hkv)]
        sa.rotate_qkv(rot, *parts, pos, *rows)
        Q, O = torch.zeros_like(rows[0]), torch.zeros_like(rows[0])
        sa.append_qkv(rot, cache.handle, *parts, pos, cu, Q)
        window, sinks = ((0, 0), (33, 2))[i % 2]
        sa.chunk_attention(cfg, cache.handle, Q, O, workspace, cu, window, sinks)
        torch.cuda.synchronize()
        got, (q, k, v) = O.double().cpu().numpy(), (r.cpu().numpy() for r in rows)
        for b in range(3):
            held[0][b], held[1][b] = (np.concatenate([h[b], r[cu[b]:cu[b + 1]]]) for h, r in zip(held, (k, v)))
            want, off = ref.attend(cfg, q[cu[b]:cu[b + 1]].astype(float), held[0][b].astype(float), held[1][b].astype(float), int(lens[b]), window, sinks)
            assert (np.abs(got[cu[b]:cu[b + 1]] - want) <= off).all(), (i, b)
        lens += new
    assert cache.seq_lens.tolist() == total.tolist()
