"""The error of the 4-bit cache's attention in the mean square, against 64 bits over the same codes: bounds that do not grow with the length, and that a
kernel without the weights' second binary16 term, or without sums of their own for a tile, does not keep (test_fp4_model.py)."""
import numpy as np
import pytest

import fp4_model as model
import fp4_reference as fp4
from paper_2609_09208_b200 import binding as sa
from paper_2609_09208_b200 import build as sa_build
from paper_2609_09208_b200 import synth
from test_fp4_model import MEAN_1
from test_gpu_fp4 import SHAPES, STREAM, attend, config, poisoned
from test_gpu_stream import marks, up

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    sa_build.build()


def check(O, Q, K, V, d, Hq, Hkv, what):
    """One sequence: outputs [Hq, d] in FP32, queries and cached numbers; all its heads together, whose values are independent of one another."""
    G, T, tile = Hq // Hkv, len(K), 64 if d == 64 else 32
    off, size, bound = 0.0, 0.0, 0.0
    for h in range(Hkv):
        q, k, v = Q[h * G:(h + 1) * G], K[:, h], V[:, h]
        want = model.exact(q, k, v)[1]
        off, size = off + ((O[h * G:(h + 1) * G] - want) ** 2).sum(), size + (want ** 2).sum()
        # (six warps at least share the tiles of a block)
        bound = max(bound, model.mean_square_bound(q, k, tile, -(-T // (6 * tile))))
    assert np.sqrt(off / size) <= bound, (what, np.sqrt(off / size), bound)


@pytest.mark.parametrize("d,Hq,Hkv,lens,room,hadamard", [(*s[:4], 0, s[4]) for s in SHAPES] + STREAM)
def test_mean_square_error_of_every_sequence(d, Hq, Hkv, lens, room, hadamard):
    import torch
    cfg = config(d, Hq, Hkv, hadamard)
    case = synth.make_case("fp4e", lens, Hq, Hkv, d, 0, outliers=True, seed=1100 + len(lens))
    c = poisoned(cfg, lens, room=room)
    c.fill(up(case.K), up(case.V), case.cu_lens)
    O = torch.full((len(lens), Hq, d), float("nan"), device="cuda")
    attend(cfg, c, up(case.Q), O)
    O = O.cpu().numpy().astype(np.float64)
    turn = fp4.hadamard if hadamard else lambda x: x
    picked = [b for b in range(len(lens)) if lens[b]]
    for b in picked[::max(1, len(picked) // 20)]:
        rows = slice(int(case.cu_lens[b]), int(case.cu_lens[b + 1]))
        check(O[b], turn(case.Q[b]), fp4.quantised(turn(case.K[rows])), fp4.quantised(case.V[rows]), d, Hq, Hkv, (b, lens[b]))


@pytest.mark.parametrize("B,T,d,Hq,Hkv", [(16, 16384, 64, 32, 4), (4, 20000, 128, 32, 8)])
def test_mean_square_error_of_long_sequences(B, T, d, Hq, Hkv):
    import torch
    cfg = config(d, Hq, Hkv)
    case = synth.make_case("fp4el", [T] * B, Hq, Hkv, d, 0, outliers=True, seed=31)
    c = sa.PagedCache(cfg, [T] * B, "cuda")
    c.fill(up(case.K), up(case.V), case.cu_lens)
    O = torch.full((B, Hq, d), float("nan"), device="cuda")
    attend(cfg, c, up(case.Q), O)
    O = O.cpu().numpy().astype(np.float64)
    for b in (0, B - 1):
        rows = slice(b * T, b * T + T)
        check(O[b], case.Q[b], fp4.quantised(case.K[rows]), fp4.quantised(case.V[rows]), d, Hq, Hkv, b)


@pytest.mark.parametrize("B,T,d,Hq,Hkv,one_per_sm", [(32, 32768, 64, 32, 4, True), (8, 32768, 128, 32, 8, True), (1, 131072, 128, 32, 8, False)])
def test_sums_over_long_stretches(B, T, d, Hq, Hkv, one_per_sm):
    """Values of mean 1, whose sums grow with every tile: 28, 37 and 18 tiles a warp.  A tile's products are cut off by up to 2^-23 of a sum that grows
    evenly over its steps: two terms of 16 keys at a time, 64 keys 5 x 2^-23 in all (2 x (1/4 + 2/4 + 3/4 + 1)), 32 keys 3 x 2^-23; 6e-7 and 3.6e-7.  The additions of
    the tiles are rounded to nearest: sqrt(37 / 3) 2^-24, 2.1e-7 at most, and the normaliser's chains, many side by side, a tenth of that.  The
    weights' own errors are independent of the values' and go down with the root of the length: 3e-6 / sqrt(10 000).  9e-7 in all: 1e-6."""
    import torch
    cfg, G, pick = config(d, Hq, Hkv), Hq // Hkv, B - 1
    gen = torch.Generator(device="cuda").manual_seed(d + B)
    c = sa.PagedCache(cfg, [T] * B, "cuda", permutation=synth.page_permutation(B * T // 64, 3))
    K = torch.randn((B * T, Hkv, d), generator=gen, device="cuda").half()
    V = (torch.randn((B * T, Hkv, d), generator=gen, device="cuda") + 1).half()
    c.fill(K, V, np.arange(B + 1) * T)
    Q = torch.randn((B, Hq, d), generator=gen, device="cuda").half()
    O = torch.full((B, Hq, d), float("nan"), device="cuda")
    c.workspace.fill_(255)
    attend(cfg, c, Q, O)
    assert (marks(c.workspace) > 0) == one_per_sm
    del K, V
    held = [torch.empty((T, Hkv, d), dtype=torch.float16, device="cuda") for _ in "kv"]      # (the cache's numbers are binary16 numbers: exact)
    starts, cu = np.zeros(B, dtype=np.int64), np.zeros(B + 1, dtype=np.int64)
    cu[pick + 1:] = T
    sa.read_kv(cfg, c.handle, starts, cu, *held)
    keys, values = (x.double() for x in held)
    q = Q[pick].double()
    want = torch.cat([torch.softmax(q[h * G:(h + 1) * G] @ keys[:, h].T / d ** 0.5, -1) @ values[:, h] for h in range(Hkv)])
    off = float((O[pick].double() - want).norm() / want.norm())
    assert off <= MEAN_1, off
