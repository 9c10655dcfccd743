"""Prompts with a common prefix, whose sequences share its pages, filled in one call: every token is there afterwards, and what lies behind
the longest is as it was."""
import numpy as np
import pytest

import fp4_reference as fp4
from paper_2609_09208_b200 import binding as sa
from paper_2609_09208_b200 import build as sa_build
from paper_2609_09208_b200 import synth

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("longest", [96, 93, 61])
@pytest.mark.parametrize("code,hadamard", [(c, h) for c in (sa.SA_KV_FP4, sa.SA_POTM4, sa.SA_POT4) for h in (False, True)] + [(sa.SA_KV_FP16, False)])
@pytest.mark.parametrize("d", [64, 128])
def test_sequences_that_end_anywhere_in_shared_pages(d, hadamard, code, longest):
    """Sequences of 1, 2, 3, ... tokens of one prompt, all on the same pages, against the longest alone.  The one that fills a half page whole,
    those that end within it and those that end at odd tokens write the same words at the same time."""
    import torch
    sa_build.build()
    H = 2
    cfg = sa.make_config(d, H, H, code, hadamard=hadamard)
    case = synth.make_case("shared", [longest], H, H, d, 0, outliers=True, seed=longest + d)
    bits = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()
    alone, shared = (sa.PagedCache(cfg, [longest], "cuda") for _ in range(2))
    alone.pages.fill_(0x5a)
    alone.fill(bits(case.K), bits(case.V), case.cu_lens)
    lens = np.concatenate([np.arange(1, longest + 1), [longest]])
    lens = lens[np.random.default_rng(d).permutation(len(lens))]
    rows = np.concatenate([np.arange(n) for n in lens])
    cu = np.concatenate([[0], np.cumsum(lens)])
    K, V = bits(case.K[rows]), bits(case.V[rows])
    table = shared.page_table.repeat(len(lens), 1).contiguous()
    seq_lens = torch.from_numpy(lens.astype(np.int32)).cuda()
    handle = sa.make_cache(shared.pages, table, seq_lens, shared.n_pages)
    for _ in range(10):
        shared.pages.fill_(0x5a)
        sa.fill_kv(cfg, handle, K, V, cu)
        torch.cuda.synchronize()
        assert torch.equal(shared.pages, alone.pages)
    if code == sa.SA_KV_FP4:
        out = [torch.zeros(len(rows), H, d, dtype=torch.float16, device="cuda") for _ in "kv"]
        sa.read_kv(cfg, handle, None, cu, *out)
        assert np.array_equal(out[1].cpu().numpy().astype(np.float64), fp4.quantised(case.V)[rows])
