"""Kernels that may start before the kernel in front of them has ended (programmatic launches) read nothing through the non-coherent
path: that is for memory which nobody writes while the kernel lives, and what such a kernel reads may be written by the one in front."""
import glob
import os
import re

import numpy as np
import pytest

from paper_2609_09208_b200 import binding as sa
from paper_2609_09208_b200 import build as sa_build

CSRC = sa_build.CSRC


def sources():
    text = {}
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cuh"))):
        with open(path) as f:
            text[os.path.basename(path)] = re.sub(r"//[^\n]*", "", f.read())
    return text


def test_no_load_asks_for_the_non_coherent_path():
    found = [(name, m.group()) for name, s in sources().items() for m in re.finditer(r"__ldg\b|ld\.global(\.\w+)*\.nc\b", s)]
    assert not found, found


def test_no_input_of_a_programmatic_launch_is_declared_read_only():
    """A `const T* __restrict__` parameter lets the compiler choose that path by itself."""
    text = "\n".join(sources().values())
    early = set(re.findall(r"launch_pdl(?:_cluster)?\(\s*(\w+_kernel)\b", text))
    assert {"append_kernel", "fill_kernel", "read_kernel", "rotate_kernel", "merge_kernel", "stage_in_kernel"} <= early
    for name in early - {"stage_in_kernel"}:       # (reads host memory, which no kernel writes, past all caches)
        declared = re.findall(r"\b%s\(([^)]*)\)\s*\{" % name, text)
        assert declared, name
        assert not any(re.search(r"const\s+\w+\s*\*\s*__restrict__", p) for p in declared), name


@pytest.mark.gpu
@pytest.mark.parametrize("code", [sa.SA_KV_FP4, sa.SA_POTM4, sa.SA_KV_FP16])
def test_a_chain_of_calls_gives_what_the_calls_one_by_one_give(code):
    """Projections -> rows -> a cache -> rows -> another cache -> rows, over and over into the same buffers with other inputs each time: the
    outputs of every round are those of a round in which each call ends before the next begins."""
    import torch
    sa_build.build()
    d, H, n = 64, 3, 517
    cfg = sa.make_config(d, H, H, code)
    caches = [sa.PagedCache(cfg, [n], "cuda") for _ in range(2)]
    cu = np.array([0, n])
    gen = torch.Generator(device="cuda").manual_seed(code)
    room = torch.empty(n * 3 * H * d + 4, device="cuda")
    inputs = [torch.randn(n, 3 * H * d, device="cuda", generator=gen) for _ in range(4)]
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    inv = (1e4 ** (-torch.arange(d // 2, device="cuda") * 2.0 / d)).float()
    rot = sa.Rotary(cfg, inv, dtype=torch.float32, norm=True)
    rows = [torch.zeros(n, H, d, dtype=torch.float16, device="cuda") for _ in range(7)]

    def round_of_calls(i, wait):
        x = room[4 * (i % 2):][:n * 3 * H * d].view(n, -1)           # on a 32-byte place and between two
        x.copy_(inputs[i % 4])
        calls = [lambda: sa.rotate_qkv(rot, *(p.unflatten(1, (H, d)) for p in x.split(H * d, 1)), pos, *rows[:3]),
                 lambda: caches[0].fill(rows[1], rows[2], cu), lambda: sa.read_kv(cfg, caches[0].handle, None, cu, *rows[3:5]),
                 lambda: caches[1].fill(rows[3], rows[4], cu), lambda: sa.read_kv(cfg, caches[1].handle, None, cu, *rows[5:7])]
        for call in calls:
            if wait:
                torch.cuda.synchronize()
            call()
        return [r.clone() for r in rows]

    want = [round_of_calls(i, True) for i in range(4)]
    assert not torch.equal(want[0][1], want[1][1])
    torch.cuda.synchronize()
    got = [round_of_calls(i, False) for i in range(60)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for i, g in enumerate(got) for a, b in zip(g, want[i % 4]))
