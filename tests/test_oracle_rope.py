"""The oracle of the heads' norm and rotation, against what has to hold of it (no GPU)."""
import numpy as np
import pytest

from oracle import rope as OR


def _inputs(R=5, H=3, d=16, h=6, seed=0):
    r = np.random.default_rng(seed)
    return (r.standard_normal((R, H, d)), 1 + 0.3 * r.standard_normal(d), r.integers(0, 5000, R),
            10000.0 ** (-np.arange(h) / max(h, 1)), r.standard_normal((R, H, d)))


def test_a_pair_is_a_complex_number_times_a_unit():
    x, w, pos, f, _ = _inputs()
    h = len(f)
    got = OR.norm_rope(x, None, pos, f, 1e-6)
    z = (x[..., :h] + 1j * x[..., h:2 * h]) * np.exp(1j * pos[:, None, None] * f)
    assert np.allclose(got[..., :h], z.real, atol=1e-12) and np.allclose(got[..., h:2 * h], z.imag, atol=1e-12)
    assert np.array_equal(got[..., 2 * h:], x[..., 2 * h:])


def test_products_depend_on_the_distance_alone_and_norms_are_one():
    x, w, _, f, _ = _inputs(R=1, H=1)
    y = np.roll(x, 3, axis=-1)
    at = lambda v, p: OR.norm_rope(v, None, [p], f, 0.0)[0, 0]
    assert np.isclose(at(x, 7) @ at(y, 3), at(x, 1007) @ at(y, 1003))
    n = OR.norm_rope(x, np.ones(16), [9], f, 0.0)
    assert np.isclose((n * n).mean(), 1.0)
    assert np.allclose(OR.norm_rope(4 * x, w, [9], f, 0.0), OR.norm_rope(x, w, [9], f, 0.0))


@pytest.mark.parametrize("weighted,h", [(True, 6), (True, 8), (True, 0), (False, 6)])
def test_gradients_against_differences(weighted, h):
    x, w, pos, f, g = _inputs(h=h)
    w = w if weighted else None
    dx, dw = OR.norm_rope_grad(x, w, pos, f, 1e-3, g)
    r = np.random.default_rng(1)
    for _ in range(5):
        v = r.standard_normal(x.shape)
        e = 1e-6
        num = ((OR.norm_rope(x + e * v, w, pos, f, 1e-3) - OR.norm_rope(x - e * v, w, pos, f, 1e-3)) * g).sum() / (2 * e)
        assert np.isclose(num, (dx * v).sum(), rtol=1e-6, atol=1e-7)
    if weighted:
        for j in (0, 7, 15):
            step = np.zeros(16)
            step[j] = 1e-6
            num = ((OR.norm_rope(x, w + step, pos, f, 1e-3) - OR.norm_rope(x, w - step, pos, f, 1e-3)) * g).sum() / 2e-6
            assert np.isclose(num, dw[j], rtol=1e-6, atol=1e-7)
