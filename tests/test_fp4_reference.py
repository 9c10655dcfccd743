"""The numpy reference of the 4-bit cache against things other than itself (no GPU)."""
import itertools

import numpy as np
import pytest

import fp4_reference as fp4


@pytest.mark.parametrize("d", [64, 128])
def test_places_fill_the_half_page_once(d):
    (k, kn), ks, (v, vn), vs = fp4.places(d)
    nibbles = np.concatenate([(2 * k + kn).ravel(), (2 * v + vn).ravel()])
    bytes_ = np.concatenate([ks[:, ::16].ravel(), vs[:, ::16].ravel()])
    assert len(set(nibbles)) == nibbles.size and len(set(bytes_)) == bytes_.size
    assert set(nibbles // 2) | set(bytes_) == set(range(36 * d)) and not set(nibbles // 2) & set(bytes_)
    assert all((ks[:, 16 * b:16 * b + 16] == ks[:, 16 * b:16 * b + 1]).all() for b in range(d // 16))


def test_scale_is_the_nearest_of_all_bytes():
    from fractions import Fraction
    grid = [Fraction(float(x)) for x in fp4.scales(np.arange(0xe3, dtype=np.uint8))]
    rng = np.random.default_rng(1)
    patterns = np.unique(np.concatenate([rng.integers(0, 0x7c00, 400), [0, 1, 2, 0x17f, 0x180, 0x181, 0x3ff, 0x400, 0x7bff, 0x2a60, 0x5260]])).astype(np.uint16)
    for p in patterns:
        amax = p.view(np.float16)
        x = np.zeros(16, np.float16)
        x[5] = -amax
        t = Fraction(float(amax)) / 6
        near = min(range(len(grid)), key=lambda i: (abs(grid[i] - t), i % 2))
        assert fp4.scale_bytes(x) == near, hex(p)


def test_codes_are_the_nearest_with_ties_to_even():
    from fractions import Fraction
    for m, e in itertools.product(range(8, 16), (-6, 0, 5)):
        s = Fraction(m) * Fraction(2) ** e
        for tie, want in [(Fraction(1, 4), 0), (Fraction(3, 4), 2), (Fraction(5, 4), 2), (Fraction(7, 4), 4), (Fraction(5, 2), 4), (Fraction(7, 2), 6), (Fraction(5), 6)]:
            x = np.zeros(16, np.float16)
            x[0] = float(6 * s)
            assert Fraction(float(x[0])) == 6 * s
            x[1], x[2] = float(tie * s), -float(tie * s)
            x[3], x[4] = np.nextafter(x[1], np.float16(0)), np.nextafter(x[1], np.float16(6e4))
            code, b = fp4.encode(x)
            assert fp4.scales(b)[0] == float(s) and code[0] == 7 and code[1] == want and code[2] == (want | 8 if want else 0)
            below = int((fp4.LEVELS < float(tie)).sum()) - 1
            assert code[3] == below and code[4] == below + 1


def test_saturation_and_flush():
    x = np.full(16, 65504, np.float16)
    assert (fp4.quantised(x) == 61440).all()
    assert not fp4.quantised(np.full(16, 6 * 2.0 ** -18, np.float16)).any()
    assert fp4.quantised(np.full(16, 6.1 * 2.0 ** -18, np.float16)).any()
