"""The bounds on the error of the 4-bit cache's attention, held against a model of its roundings (no GPU): the kernels' form keeps them; a
form without the weights' second binary16 term, or without sums of their own for a tile, does not."""
import numpy as np
import pytest

import fp4_model as model
import fp4_reference as fp4
from paper_2609_09208_b200 import synth

MEAN_1 = 1e-6          # of outputs over values of mean 1 (derived in test_gpu_fp4_error.py)


def inputs(d, G, T, outliers=True, mean=0.0):
    c = synth.make_case("model", [T], G, 1, d, 0, outliers=outliers, seed=5 + T)
    return c.Q[0], fp4.quantised(c.K)[:, 0], fp4.quantised((c.V[:, 0].astype(np.float32) + mean).astype(np.float16))


def off(o, want):
    return np.sqrt(((o - want) ** 2).mean() / (want ** 2).mean())


def test_cut():
    x = np.array([1.0 + 2.0 ** -24, -1.0 - 3 * 2.0 ** -25, 1.0 - 2.0 ** -25, 0.0, 2.0 ** 20 + 1.0])
    assert np.array_equal(model.cut(x), np.array([1.0, -1.0, 1.0 - 2.0 ** -24, 0.0, 2.0 ** 20 + 1.0], np.float32))


@pytest.mark.parametrize("d,G,T,outliers,tile,chains", [(64, 8, 16384, True, 64, 24), (64, 8, 4096, False, 64, 12), (128, 4, 20000, True, 32, 48),
                                                        (64, 8, 700, True, 64, 6), (64, 1, 200, True, 64, 6), (128, 7, 333, False, 32, 6)])
def test_the_second_term_of_a_weight_shows(d, G, T, outliers, tile, chains):
    q, k, v = inputs(d, G, T, outliers)
    _, want = model.exact(q, k, v)
    bound = model.mean_square_bound(q, k, tile, -(-T // (6 * tile)))
    full, one = (off(model.attention(q, k, v, tile=tile, chains=chains, terms=n), want) for n in (2, 1))
    assert full <= bound < one / 10, (full, bound, one)


@pytest.mark.parametrize("d,G,tile,tiles", [(64, 8, 64, 28), (128, 4, 32, 37), (128, 4, 32, 18)])
def test_sums_of_their_own_for_a_tile_show(d, G, tile, tiles):
    q, k, v = inputs(d, G, tiles * tile * 4, False, 1.0)
    _, want = model.exact(q, k, v)
    own, joined = (off(model.attention(q, k, v, tile=tile, chains=4, fine=fine), want) for fine in (True, False))
    assert own <= MEAN_1 < joined, (own, joined)
