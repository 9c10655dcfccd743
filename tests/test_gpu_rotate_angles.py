"""sa_rotate_qkv: the turn of a pair of which one channel is zero, where an error of the sine stands alone."""
import numpy as np
import pytest

from paper_2609_09208_b200 import binding as sa
from paper_2609_09208_b200 import build as sa_build

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("d,kind", [(64, "float32"), (128, "bfloat16"), (64, "float16")])
def test_sine_and_cosine_to_their_last_bits(d, kind, neighbours):
    """Channels (0, b) become (-b sin, b cos), and (a, 0) (a cos, a sin): products of one number, so the error is relative to the output.  One rounding
    to binary16, 2^-11; before it 32-bit steps: the fraction of a turn 2^-24, sine or cosine 2^-23, the two products 2^-24 each, and
    where an angle is beyond an eighth of a turn the fraction's rounding as an angle, 2^-24 of it: pi 2^-24 at most next to a zero of sine or cosine."""
    import torch
    sa_build.build()
    t, n = getattr(torch, kind), 1200
    inv = np.exp(np.linspace(np.log(1.0), np.log(1e-7), d // 2)).astype(np.float32)
    pos = np.concatenate([np.arange(200), np.arange(-200, 0), 1 << np.arange(20), np.random.default_rng(d).integers(0, 1 << 20, n - 420)]).astype(np.int32)
    x = torch.randn(n, 2, d // 2, generator=torch.Generator().manual_seed(d)).to(t)
    j = np.arange(d // 2)
    first, second = (2 * j, 2 * j + 1) if neighbours else (j, j + d // 2)
    Q = torch.zeros(n, 2, d, dtype=t)
    Q[:, 0, second], Q[:, 1, first] = x[:, 0], x[:, 1]
    rot = sa.Rotary(sa.make_config(d, 2, 1, sa.SA_POTM4), torch.from_numpy(inv).cuda(), dtype=t, pairs="neighbours" if neighbours else "halves", scale=1.5)
    out = torch.zeros(n, 2, d, dtype=torch.float16, device="cuda")
    sa.rotate_qkv(rot, Q.cuda(), None, None, torch.from_numpy(pos).cuda(), out, None, None)
    out, x = out.double().cpu().numpy(), 1.5 * x.double().numpy()
    angle = pos.astype(np.float64)[:, None] * inv.astype(np.float64)
    c, s = np.cos(angle), np.sin(angle)
    for got, b, f in ((out[:, 0, first], -x[:, 0], s), (out[:, 0, second], x[:, 0], c), (out[:, 1, first], x[:, 1], c), (out[:, 1, second], x[:, 1], s)):
        want = b * f
        far = np.minimum(np.abs(angle), np.pi) * 2.0 ** -24 * np.abs(b) + 2.0 ** -50 * np.abs(angle * b)
        tol = np.maximum(np.abs(want) * 2.0 ** -11, 2.0 ** -25) + 6 * 2.0 ** -24 * np.abs(want) + far * (np.abs(angle) > 0.78)
        assert (np.abs(got - want) <= tol).all(), np.max(np.abs(got - want) / tol)
