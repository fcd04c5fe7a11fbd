"""The oracle of the paged cache against torch's e4m3 and against what can be counted by hand."""
import numpy as np
import pytest

from oracle import paged as OP


def test_e4m3_is_torchs():
    import torch
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy().astype(np.float64)
    fine = ~np.isnan(every)
    assert np.array_equal(OP.e4m3(every[fine]), every[fine])
    assert np.array_equal(OP.e4m3_byte(every[fine]), np.arange(256, dtype=np.uint8)[fine])
    r = np.random.default_rng(0)
    x = np.concatenate([r.standard_normal(20000) * 10.0 ** r.uniform(-4, 2, 20000), (every[fine][:-1] + every[fine][1:]) / 2])
    x = np.float64(np.float32(x[np.abs(x) <= 448]))
    assert np.array_equal(OP.e4m3(x), torch.from_numpy(np.float32(x)).to(torch.float8_e4m3fn).float().numpy().astype(np.float64))
    assert np.isnan(OP.e4m3([np.nan, np.inf, -np.inf])).all() and OP.e4m3_byte(np.nan) == 0x7f


@pytest.mark.parametrize("most,s", [(448.0, 1.0), (448.0001, 2.0), (224.0, 0.5), (1.0, 2.0 ** -8), (0.0, 2.0 ** -120), (1e-40, 2.0 ** -120), (3.4e38, 2.0 ** 120)])
def test_scale(most, s):
    assert OP.scale_for([most, -most / 3, np.nan, np.inf]) == s


def test_rounding_again_loses_nothing_above_the_least_exponent():
    # the scale grows eightfold: entries above 2^-6 of the new scale keep their value
    r = np.random.default_rng(1)
    a = OP.Sequence(1, 64)
    first = r.uniform(0.25, 1.0, (3, 1, 64))
    a.append(first)
    before = a.numbers()
    a.append(np.full((2, 1, 64), 8.0))
    assert a.scales[0, 0] == 2.0 ** -5 and np.array_equal(a.numbers()[:3], before)
    # dropped to the block's start: the scale starts anew; in its middle it stays
    a.append(np.full((1, 1, 64), 0.5), keep=2)
    assert len(a) == 3 and a.scales[0, 0] == 2.0 ** -5 and np.array_equal(a.numbers()[:2], before[:2])
    a.append(np.full((1, 1, 64), 0.5), keep=0)
    assert len(a) == 1 and a.scales[0, 0] == 2.0 ** -9


def test_places_are_a_page():
    for d in (64, 128):
        r, x = np.meshgrid(np.arange(32), np.arange(d), indexing="ij")
        for place in (OP.key_place, OP.value_place):
            assert sorted(place(r, x, d).ravel()) == list(range(32 * d))
        # sixteen bytes of a key in a row, four keys' bytes of a value element in a word
        assert list(OP.key_place(5, np.arange(16, 32), d) - OP.key_place(5, 16, d)) == list(range(16))
        assert list(OP.value_place(np.arange(4, 8), 9, d) - OP.value_place(4, 9, d)) == [0, 1, 2, 3]
