"""The oracle of sampling, against what has to hold of it (no GPU)."""
import numpy as np
import pytest

from oracle import sample as OS


def test_written_out_by_hand():
    z = np.log([1.0, 4.0, 2.0, 4.0, 5.0])
    ids = lambda **kw: OS.kept_weights(z, 1.0, **kw)[0].tolist()
    assert ids() == [4, 1, 3, 2, 0]
    assert ids(top_k=2) == [4, 1] and ids(top_k=9) == [4, 1, 3, 2, 0]
    # weights 5 4 4 2 1 of 16; in front of them 0 5 9 13 15
    assert ids(top_p=0.5) == [4, 1] and ids(top_p=0.6) == [4, 1, 3] and ids(top_p=0.0) == [4] and ids(top_p=9 / 16 + 1e-9) == [4, 1, 3]
    assert ids(top_k=3, top_p=0.7) == [4, 1, 3] and ids(top_k=3, top_p=0.69) == [4, 1]
    assert ids(min_p=0.5) == [4, 1, 3] and ids(min_p=1.0) == [4] and ids(min_p=7.0) == [4] and ids(min_p=0.39) == [4, 1, 3, 2]
    assert [OS.sample(z, u)[0] for u in (0.0, 0.3, 0.32, 0.6, 0.9, 0.99)] == [4, 4, 1, 3, 2, 0]
    assert OS.sample(z, 0.9, temperature=0)[0] == 4


@pytest.mark.parametrize("kw", [dict(), dict(top_k=3), dict(top_p=0.8), dict(min_p=0.2), dict(temperature=0.5, top_k=5, top_p=0.9)])
def test_shares_of_many_draws(kw):
    r = np.random.default_rng(0)
    z = r.standard_normal(8)
    ids, w = OS.kept_weights(z, kw.get("temperature", 1.0), **{k: v for k, v in kw.items() if k != "temperature"})
    n = 4000
    got = np.bincount([OS.sample(z, (i + 0.5) / n, **kw)[0] for i in range(n)], minlength=8) / n
    want = np.zeros(8)
    want[ids] = w / w.sum()
    assert np.abs(got - want).max() <= 1.0 / n
