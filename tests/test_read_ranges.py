"""sa_read_kv at the end of the longest caches: positions up to 2^31 - 1."""
import ctypes as C
import os
import subprocess
import sys

import numpy as np
import pytest

import fp4_reference as fp4
from paper_2609_09208_b200 import binding as sa
from paper_2609_09208_b200 import build as sa_build
from paper_2609_09208_b200 import synth

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
END = (1 << 31) - 1                                # lengths are 32-bit numbers
PAGES = 1 << 25                                    # room for one token more


@pytest.fixture(scope="module", autouse=True)
def _built():
    sa_build.build()


def test_half_pages_up_to_the_last_token_are_counted():
    """Three sequences: the last token of all, and two ranges of 2^26 - 1 half pages.  Added up in 32 bits the first came out as
    -2 (2^26 - 1) half pages, the three as none, and the call as a success that had read nothing.  Without a GPU (in a process that sees
    none) a call that goes as far as its launch comes back with status 5."""
    call = """
import ctypes as C
from paper_2609_09208_b200 import binding as sa
cfg, cache, at = sa.make_config(64, 1, 1, sa.SA_KV_FP4), sa.SaCache(256, 256, 256, 3, %d, 8), C.c_void_p(256)
n = 32 * ((1 << 26) - 1)
i64 = lambda *v: (C.c_int64 * len(v))(*v)
print(sa.lib().sa_read_kv(C.byref(cfg), C.byref(cache), i64(%d, 0, 0), i64(0, 1, 1 + n, 1 + 2 * n), at, None, None))
""" % (PAGES, END - 1)
    run = subprocess.run([sys.executable, "-c", call], cwd=ROOT, capture_output=True, text=True, env={**os.environ, "CUDA_VISIBLE_DEVICES": ""}, timeout=600)
    assert run.returncode == 0 and run.stdout.split() == ["5"], run.stdout + run.stderr


def test_a_read_of_no_tokens_needs_no_outputs():
    """A tensor without elements has no address: a read of no tokens into two of them is not one without outputs.  What else is wrong with
    such a call is said all the same."""
    lib, i64, at, null = sa.lib(), lambda *v: (C.c_int64 * len(v))(*v), C.c_void_p(256), C.c_void_p(0)
    cfg, cache = sa.make_config(64, 32, 4, sa.SA_KV_FP4), sa.SaCache(256, 256, 256, 2, 4, 8)
    call = lambda cu, starts, K, V: lib.sa_read_kv(C.byref(cfg), C.byref(cache), starts, cu, K, V, null)
    for K, V in ((null, null), (at, null), (null, at), (at, at)):
        assert call(i64(0, 0, 0), None, K, V) == 0 and call(i64(7, 7, 7), i64(256, 3), K, V) == 0
        assert call(i64(0, 0, 0), i64(257, 0), K, V) == 4 and call(i64(0, 0, 0), i64(-1, 0), K, V) == 1
    assert call(i64(0, 0, 1), None, null, null) == 1


@pytest.mark.gpu
def test_a_read_of_no_tokens_into_empty_tensors():
    import torch
    cfg = sa.make_config(64, 4, 4, sa.SA_POTM4)
    c = sa.PagedCache(cfg, [10, 0], "cuda")
    none = torch.empty(0, 4, 64, dtype=torch.float16, device="cuda")
    sa.read_kv(cfg, c.handle, None, np.array([0, 0, 0]), none, none)
    sa.read_kv(cfg, c.handle, np.array([10, 0]), np.array([0, 0, 0]), None, none)


@pytest.mark.gpu
@pytest.mark.parametrize("hadamard", [False, True])
def test_a_range_that_ends_with_the_last_token(hadamard):
    """A page table of 2^25 pages of which the last is mapped: zeros from the page before it, and its tokens but the last."""
    import torch
    cfg = sa.make_config(64, 2, 2, sa.SA_KV_FP4, hadamard=hadamard)
    case = synth.make_case("end", [64], 2, 2, 64, 0, seed=21)
    bits = lambda x: torch.from_numpy(x).cuda()
    small = sa.PagedCache(cfg, [64], "cuda")
    small.fill(bits(case.K), bits(case.V), case.cu_lens)
    whole = [torch.zeros(64, 2, 64, dtype=torch.float16, device="cuda") for _ in "kv"]
    sa.read_kv(cfg, small.handle, None, case.cu_lens, *whole)
    table = torch.full((1, PAGES), -1, dtype=torch.int32, device="cuda")
    table[0, -1] = small.page_table[0, 0]
    far = sa.make_cache(small.pages, table, small.seq_lens, small.n_pages)
    start = 64 * (PAGES - 1) - 10
    out = [torch.full((75, 2, 64), 3.0, dtype=torch.float16, device="cuda") for _ in "kv"]
    sa.read_kv(cfg, far, np.array([start]), np.array([1, 74]), *out)
    torch.cuda.synchronize()
    assert start + 73 == END
    for o, w in zip(out, whole):
        assert not o[1:11].any() and torch.equal(o[11:74], w[:63]) and bool((o[0] == 3).all()) and bool((o[74] == 3).all())
    if not hadamard:
        assert np.array_equal(whole[0].cpu().numpy(), fp4.quantised(case.K))
    for n in (74, 75):                             # one token more, two
        with pytest.raises(sa.SaError) as err:
            sa.read_kv(cfg, far, np.array([start]), np.array([0, n]), *[torch.empty(n, 2, 64, dtype=torch.float16, device="cuda") for _ in "kv"])
        assert err.value.status == 4
