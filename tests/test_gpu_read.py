"""sa_read_kv: keys and values back out of caches of every code and container."""
import numpy as np
import pytest

import fp4_reference as fp4
from paper_2609_09208_b200 import binding as sa
from paper_2609_09208_b200 import build as sa_build
from paper_2609_09208_b200 import synth
from test_gpu_stream import up

pytestmark = pytest.mark.gpu
CODES = [(sa.SA_POT4, False), (sa.SA_POT4, True), (sa.SA_POTM1, False), (sa.SA_POTM1, True), (sa.SA_POTM2, False), (sa.SA_POTM2, True),
         (sa.SA_POTM4, False), (sa.SA_INT8, False), (sa.SA_KV_FP16, False), (sa.SA_KV_FP4, False)]
LENS = [0, 1, 31, 33, 64, 65, 130, 7]


@pytest.fixture(scope="module", autouse=True)
def _built():
    sa_build.build()


def stored(cfg, c, code, K, V, lens):
    """What the cache holds, in 64 bits, in the rotated space where keys are rotated: [tokens, KV head, d]."""
    import torch
    if code == sa.SA_KV_FP16:
        return K.astype(np.float64), V.astype(np.float64)
    if code == sa.SA_KV_FP4:
        return fp4.quantised(fp4.hadamard(K) if cfg.flags & 1 else K), fp4.quantised(V)
    Ks, Vs = [], []
    for b, n in enumerate(lens):
        shape = (n, cfg.n_kv_heads)
        codes = torch.zeros(*shape, cfg.head_dim, dtype=torch.uint8, device="cuda")
        v_hat, g = torch.zeros_like(codes).view(torch.int8), torch.zeros(shape, dtype=torch.int8, device="cuda")
        scale = torch.zeros(shape, dtype=torch.float16, device="cuda")
        if n:
            sa.debug_unpack(cfg, c.handle, b, n, codes, scale, v_hat, g)
        codes, scale, v_hat, g = (x.cpu().numpy() for x in (codes, scale, v_hat, g))
        s = scale.astype(np.float64)[..., None]
        if code == sa.SA_INT8:
            k = codes.view(np.int8) * s / 127.0
        else:
            e = (codes >> 4 & 7).astype(np.float64)
            k = np.where(e == 7, 0.0, (1 + (codes & 15) / 16.0) * 2.0 ** -e) * np.where(codes & 128, -1.0, 1.0) * s
        Ks.append(k)
        Vs.append(v_hat * 2.0 ** -g.astype(np.float64)[..., None])
    return np.concatenate(Ks), np.concatenate(Vs)


def half_step(x):
    """Half a step of binary16 at x, 2^-25 in the subnormal range."""
    return np.maximum(np.abs(x) * 2.0 ** -11, 2.0 ** -25)


@pytest.mark.parametrize("d,Hkv", [(64, 4), (128, 3)])
@pytest.mark.parametrize("code,dense,hadamard", [(*c, h) for c in CODES for h in (False, True) if c[0] != sa.SA_KV_FP16 or not h])      # (binary16 is never rotated)
def test_reads_what_the_codes_stand_for(code, dense, d, Hkv, hadamard):
    """Whole sequences and ranges from odd places; rows that are not asked for, and rows behind the last, stay."""
    import torch
    cfg = sa.make_config(d, Hkv, Hkv, code, nibble=dense, hadamard=hadamard)
    case = synth.make_case("read", LENS, Hkv, Hkv, d, 0, outliers=True, seed=d + code)
    case.V[::5] *= np.float16(1e-5)
    n_pages = int(np.maximum((case.lens + 63) // 64, 1).sum())
    c = sa.PagedCache(cfg, case.lens, "cuda", permutation=synth.page_permutation(n_pages, 3))
    c.pages.fill_(0xff)
    c.fill(up(case.K), up(case.V), case.cu_lens)
    K, V = stored(cfg, c, code, case.K, case.V, LENS)
    tol_K = half_step(K) * (1 + 1e-3)
    if hadamard:
        # in 32 bits: log2(d) + 1 roundings of numbers no larger than the sum of magnitudes
        H = np.array([[(-1.0) ** bin(i & j).count("1") for j in range(d)] for i in range(d)]) / np.sqrt(d)
        reach = np.abs(K).sum(-1, keepdims=True) / np.sqrt(d)
        K = K @ H
        tol_K = half_step(K) * (1 + 1e-3) + 9 * 2.0 ** -24 * reach
    tol_V = half_step(V) * (1 + 1e-3)
    for starts, counts in [(None, LENS), ([0, 0, 5, 31, 63, 1, 40, 7], [0, 1, 20, 2, 1, 64, 80, 0]), ([0, 1, 31, 0, 33, 65, 129, 3], [0, 0, 0, 33, 31, 0, 1, 4])]:
        cu = np.concatenate([[2], 2 + np.cumsum(counts)])
        starts = None if starts is None else np.array(starts)
        rows = np.concatenate([case.cu_lens[b] + (0 if starts is None else starts[b]) + np.arange(n) for b, n in enumerate(counts)]).astype(np.int64)
        out = [torch.full((int(cu[-1]) + 3, Hkv, d), 777.0, dtype=torch.float16, device="cuda") for _ in range(4)]
        sa.read_kv(cfg, c.handle, starts, cu, out[0], out[1])
        sa.read_kv(cfg, c.handle, starts, cu, out[2], None)
        sa.read_kv(cfg, c.handle, starts, cu, None, out[3])
        torch.cuda.synchronize()
        assert torch.equal(out[0], out[2]) and torch.equal(out[1], out[3])
        for got, want, tol in ((out[0], K, tol_K), (out[1], V, tol_V)):
            got = got.cpu().numpy().astype(np.float64)
            assert (np.abs(got[2:int(cu[-1])] - want[rows]) <= tol[rows]).all()
            assert (got[:2] == 777).all() and (got[int(cu[-1]):] == 777).all()


@pytest.mark.parametrize("code", [sa.SA_KV_FP4, sa.SA_POTM4])
def test_unmapped_pages_read_as_zeros(code):
    import torch
    cfg = sa.make_config(64, 2, 2, code)
    case = synth.make_case("readu", [200], 2, 2, 64, 0, seed=5)
    c = sa.PagedCache(cfg, [200], "cuda")
    c.fill(up(case.K), up(case.V), case.cu_lens)
    whole, holes = ([torch.full((200, 2, 64), 3.0, dtype=torch.float16, device="cuda") for _ in "kv"] for _ in range(2))
    sa.read_kv(cfg, c.handle, None, np.array([0, 200]), *whole)
    c.page_table[0, 1], c.page_table[0, 3] = -1, 1 << 20
    sa.read_kv(cfg, c.handle, None, np.array([0, 200]), *holes)
    torch.cuda.synchronize()
    for w, h in zip(whole, holes):
        assert torch.equal(h[:64], w[:64]) and torch.equal(h[128:192], w[128:192]) and not h[64:128].any() and not h[192:].any()


def test_many_sequences_and_a_captured_call():
    import torch
    lens = np.array([(29 * i) % 70 for i in range(150)])
    cfg = sa.make_config(64, 4, 4, sa.SA_KV_FP4)
    case = synth.make_case("readm", lens, 4, 4, 64, 0, seed=6)
    c = sa.PagedCache(cfg, lens, "cuda", permutation=synth.page_permutation(int(np.maximum((lens + 63) // 64, 1).sum()), 8))
    K, V = (torch.full((len(case.K), 4, 64), 3.0, dtype=torch.float16, device="cuda") for _ in "kv")
    Kin, Vin = up(case.K), up(case.V)
    c.fill(Kin, Vin, case.cu_lens)
    sa.read_kv(cfg, c.handle, None, case.cu_lens, K, V)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sa.fill_kv(cfg, c.handle, Kin, Vin, case.cu_lens)
        sa.read_kv(cfg, c.handle, None, case.cu_lens, K, V)
    for flip in (1, -1):
        Kin.copy_(up((case.K.astype(np.float32) * flip).astype(np.float16)))
        K.fill_(3)
        c.pages.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(K.cpu().numpy().astype(np.float64), flip * fp4.quantised(case.K)) and np.array_equal(V.cpu().numpy().astype(np.float64), fp4.quantised(case.V))


@pytest.mark.parametrize("hadamard", [False, True])
def test_rows_that_start_between_32_byte_places(hadamard):
    """Tensors on 16-byte boundaries only, in and out: the same bytes as from aligned ones."""
    import torch
    cfg, n = sa.make_config(64, 3, 3, sa.SA_KV_FP4, hadamard=hadamard), 77
    case = synth.make_case("reado", [n], 3, 3, 64, 0, seed=9)
    room = n * 3 * 64
    aligned = [up(case.K).view(torch.float16), up(case.V).view(torch.float16)]
    shifted = [torch.empty(room + 8, dtype=torch.float16, device="cuda")[8:].view(n, 3, 64) for _ in range(4)]
    for s, a in zip(shifted, aligned):
        s.copy_(a.view(n, 3, 64))
        assert s.data_ptr() % 32 == 16
    caches = [sa.PagedCache(cfg, [n], "cuda") for _ in range(2)]
    caches[0].fill(*aligned, case.cu_lens)
    caches[1].fill(*shifted[:2], case.cu_lens)
    out = [torch.zeros(n, 3, 64, dtype=torch.float16, device="cuda") for _ in "kv"]
    sa.read_kv(cfg, caches[0].handle, None, case.cu_lens, *out)
    sa.read_kv(cfg, caches[1].handle, None, case.cu_lens, *shifted[2:])
    torch.cuda.synchronize()
    assert torch.equal(caches[0].pages, caches[1].pages) and torch.equal(out[0], shifted[2]) and torch.equal(out[1], shifted[3])


def test_rows_beyond_32_bits():
    """A row whose place in the output is beyond 2^32 bytes and 2^31 elements."""
    import torch
    cfg, row = sa.make_config(64, 1, 1, sa.SA_KV_FP4), (1 << 25) + 5
    case = synth.make_case("readb", [90], 1, 1, 64, 0, seed=10)
    c = sa.PagedCache(cfg, [90], "cuda")
    c.fill(up(case.K), up(case.V), case.cu_lens)
    K = torch.zeros(row + 90, 1, 64, dtype=torch.float16, device="cuda")
    assert row * 64 > 1 << 31
    sa.read_kv(cfg, c.handle, None, np.array([row, row + 90]), K, None)
    assert np.array_equal(K[row:].cpu().numpy(), fp4.quantised(case.K)) and not K[:row].any()
    del K
    torch.cuda.empty_cache()


def test_what_is_read_can_be_written_again():
    """A 4-bit cache read out and written again holds the same numbers where the largest of every block is its scale's 6."""
    import torch
    cfg = sa.make_config(128, 2, 2, sa.SA_KV_FP4)
    case = synth.make_case("again", [300], 2, 2, 128, 0, seed=7)
    case.K[..., ::16], case.V[..., ::16] = 6.0, -12.0
    case.K[:], case.V[:] = np.clip(case.K, -6, 6), np.clip(case.V, -12, 12)
    c = sa.PagedCache(cfg, [300], "cuda")
    c.fill(up(case.K), up(case.V), case.cu_lens)
    out = [torch.full((300, 2, 128), 3.0, dtype=torch.float16, device="cuda") for _ in range(4)]
    sa.read_kv(cfg, c.handle, None, np.array([0, 300]), out[0], out[1])
    c.pages.fill_(0xff)
    c.fill(out[0], out[1], case.cu_lens)
    sa.read_kv(cfg, c.handle, None, np.array([0, 300]), out[2], out[3])
    torch.cuda.synchronize()
    assert torch.equal(out[0], out[2]) and torch.equal(out[1], out[3])


def test_the_binding_refuses_what_does_not_fit():
    import torch
    cfg = sa.make_config(64, 4, 4, sa.SA_KV_FP4)
    c = sa.PagedCache(cfg, [100, 100], "cuda")
    good = torch.zeros(200, 4, 64, dtype=torch.float16, device="cuda")
    call = lambda K, V=None, starts=None, cu=(0, 100, 200): sa.read_kv(cfg, c.handle, None if starts is None else np.array(starts), np.array(cu), K, V)
    call(good)
    for bad in (good[:199], good.float(), good.cpu(), good.view(200, 2, 128), torch.zeros(200, 4, 128, dtype=torch.float16, device="cuda")[..., :64],
                torch.zeros(400, 4, 64, dtype=torch.float16, device="cuda")[::2], good[0]):
        with pytest.raises(ValueError):
            call(bad)
        with pytest.raises(ValueError):
            call(None, bad)
    with pytest.raises(ValueError, match="starts"):
        call(good, starts=[0])
    for cu in (np.array([0, 1, 2], dtype=np.int32), np.array([0.0, 1.0, 2.0]), np.array([0, 9, 1, 9, 2])[::2], np.array([0, 1])):
        with pytest.raises(ValueError):
            sa.read_kv(cfg, c.handle, None, cu, good, None)
    for starts, cu, status in ((None, (0, 100, 50), 1), ([-1, 0], (0, 1, 2), 1), ([100, 0], (0, 29, 30), 4), ([129, 0], (0, 0, 1), 4), (None, (0, 129, 130), 4)):
        with pytest.raises(sa.SaError) as err:
            call(good, starts=starts, cu=cu)
        assert err.value.status == status, (starts, cu)
    with pytest.raises(sa.SaError):
        call(None)
