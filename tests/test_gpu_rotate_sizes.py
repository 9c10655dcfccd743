"""sa_rotate_qkv: prompts of more tokens than a position grid of 131 072, few heads."""
import numpy as np
import pytest

from paper_2609_09208_b200 import binding as sa
from paper_2609_09208_b200 import build as sa_build
from test_gpu_rotate import frequencies, reference, tolerance

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,R,neighbours,axes,norm,n", [("float16", 64, False, 1, False, 349525), ("bfloat16", 32, False, 3, True, 131072),
                                                           ("float32", 48, True, 2, True, 200001)])
def test_long_prompts_of_one_head(kind, R, neighbours, axes, norm, n):
    """1 / 1 heads of 64, queries, keys and values side by side: sampled tokens, the first and the last against the formulas, values all."""
    import torch
    sa_build.build()
    d, t = 64, getattr(torch, kind)
    gen = torch.Generator(device="cuda").manual_seed(n)
    x = torch.randn(n, 3 * d, device="cuda", generator=gen).to(t)
    pos = torch.randint(0, 1 << 20, (axes, n), generator=gen, device="cuda", dtype=torch.int32)
    axis = (torch.arange(R // 2) % axes).byte()
    w = [(1 + 0.3 * torch.randn(d, device="cuda", generator=gen)).to(t) if norm else None for _ in "qk"]
    rot = sa.Rotary(sa.make_config(d, 1, 1, sa.SA_KV_FP4), torch.from_numpy(frequencies(R)).cuda(), dtype=t, pairs="neighbours" if neighbours else "halves",
                    n_axes=axes, pair_axis=axis.cuda() if axes > 1 else None, norm=norm, eps=1e-5, q_weight=w[0], k_weight=w[1])
    outs = [torch.full((n + 1, 1, d), 777.0, dtype=torch.float16, device="cuda") for _ in range(3)]
    parts = [v.unflatten(1, (1, d)) for v in x.split(d, 1)]
    sa.rotate_qkv(rot, *parts, pos, *[o[:n] for o in outs])
    rows = np.unique(np.concatenate([np.random.default_rng(n).integers(0, n, 3000), np.arange(9), n - 1 - np.arange(9)]))
    at = torch.from_numpy(rows).cuda()
    for i in range(2):
        y, size = reference(parts[i][at].double().cpu().numpy(), R, neighbours, pos[:, at].cpu().numpy(), axis.long().numpy() * (axes > 1), frequencies(R),
                            norm, 1e-5, None if w[i] is None else w[i].double().cpu().numpy(), 1.0)
        assert (np.abs(outs[i][at].double().cpu().numpy() - y) <= tolerance(y, size)).all()
    assert torch.equal(outs[2][:n], parts[2].half()) and all(bool((o[n] == 777).all()) for o in outs)
