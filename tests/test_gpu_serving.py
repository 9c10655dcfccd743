"""A serving loop over a power-of-two cache, from a layer's projections to outputs: each step's outputs against the oracle, at the tolerance that
tells a step that left its own token out."""
import numpy as np
import pytest

from oracle import sa_oracle as ora
from paper_2609_09208_b200 import binding as sa
from paper_2609_09208_b200 import build as sa_build
from test_gpu_parity import E, TOL_O

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("code,dense,hadamard", [(sa.SA_POTM4, False, False), (sa.SA_POTM4, False, True), (sa.SA_POT4, True, False), (sa.SA_POTM2, True, False)])
def test_steps_from_projections_against_the_oracle(code, dense, hadamard):
    """Prompts of 70, 5 and no tokens, then 5 tokens each, the step captured once and replayed."""
    import torch
    sa_build.build()
    d, Hq, Hkv, n = 64, 8, 2, 5
    lens = np.array([70, 5, 0])
    B, wide = len(lens), (Hq + 2 * Hkv) * d
    gen = torch.Generator().manual_seed(40 + code)
    cfg = sa.make_config(d, Hq, Hkv, code, nibble=dense, hadamard=hadamard)
    w = [(1 + 0.2 * torch.randn(d, generator=gen)).bfloat16().cuda() for _ in "qk"]
    inv = torch.from_numpy((1e4 ** (-np.arange(d // 2) * 2.0 / d)).astype(np.float32)).cuda()
    rot = sa.Rotary(cfg, inv, dtype=torch.bfloat16, norm=True, q_weight=w[0], k_weight=w[1])
    cache = sa.PagedCache(cfg, lens, "cuda", extra_tokens=n)
    parts = lambda x: [v.unflatten(1, (-1, d)) for v in x.split([Hq * d, Hkv * d, Hkv * d], 1)]
    rows = lambda k: [torch.zeros(k, h, d, dtype=torch.float16, device="cuda") for h in (Hq, Hkv, Hkv)]
    cu = np.concatenate([[0], np.cumsum(lens)])
    prompt = rows(int(cu[-1]))
    where = torch.from_numpy(np.concatenate([np.arange(k) for k in lens]).astype(np.int32)).cuda()
    sa.rotate_qkv(rot, *parts(torch.randn(int(cu[-1]), wide, generator=gen).bfloat16().cuda()), where, *prompt)
    cache.fill(prompt[1], prompt[2], cu)
    x, pos, new, O = torch.zeros(B, wide, dtype=torch.bfloat16, device="cuda"), cache.seq_lens.clone(), rows(B), torch.full((B, Hq, d), float("nan"), device="cuda")

    def step():
        pos.copy_(cache.seq_lens)
        sa.rotate_qkv(rot, *parts(x), pos, *new)
        sa.decode_step(cfg, cache.handle, *new, O, cache.workspace)

    held = [[prompt[i].cpu().numpy()[cu[b]:cu[b + 1]] for b in range(B)] for i in (1, 2)]
    graph = None
    for i in range(n):
        x.copy_(torch.randn(B, wide, generator=gen).bfloat16())
        if i == 1:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        graph.replay() if graph else step()
        torch.cuda.synchronize()
        q, k, v = (t.cpu().numpy() for t in new)
        before = [np.concatenate(h) for h in held]
        held = [[np.concatenate([h[b], t[b:b + 1]]) for b in range(B)] for h, t in zip(held, (k, v))]
        now = [np.concatenate(h) for h in held]
        attention = lambda kv, length: ora.decode_attention(q, *kv, np.concatenate([[0], np.cumsum(length)]).astype(np.int64), code, E + code, hadamard=hadamard)["O"]
        want = attention(now, lens + i + 1)
        got = O.cpu().numpy()
        assert np.isfinite(got).all() and np.abs(got - want).max() <= TOL_O, (i, np.abs(got - want).max())
        some = lens + i > 0                         # (without its own token the first step of an empty sequence has none)
        without = attention(before, lens + i)
        # what the tolerance is for: every sequence's outputs would be further off without the newest token
        assert (np.abs(without - want).max((1, 2)) > 10 * TOL_O)[some].all()
    assert np.array_equal(cache.seq_lens.cpu().numpy(), lens + n)
