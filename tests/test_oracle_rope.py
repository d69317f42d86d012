"""The oracle's rotation against complex numbers, its gradients against differences, its eviction against a plain walk."""
import numpy as np
import pytest

from oracle import skipffn_oracle as O


def setting(rot, D, axes=1, T=5, H=3, seed=0):
    rng = np.random.default_rng(seed)
    pos = rng.integers(-1000, 100000, (axes, T))
    freq = 10000.0 ** (-np.arange(rot // 2) * 2 / max(rot, 1))
    axis = rng.integers(0, axes, rot // 2)
    return rng, rng.standard_normal((T, H, D)), O.rope_angles(pos, freq, axis)


@pytest.mark.parametrize("rot,D", [(16, 16), (8, 24), (0, 8)])
@pytest.mark.parametrize("neighbours", [False, True])
def test_pairs_turn_as_complex_numbers(rot, D, neighbours):
    _, x, angle = setting(rot, D, 3)
    y, n = O.rope_forward_real(x, angle, neighbours, False, None, 0.0)
    a, b = O.rope_pairs(rot, neighbours)
    z = (x[..., a] + 1j * x[..., b]) * np.exp(1j * angle)[:, None]
    assert np.allclose(y[..., a], z.real, atol=1e-12) and np.allclose(y[..., b], z.imag, atol=1e-12)
    assert np.array_equal(y[..., rot:], x[..., rot:]) and np.array_equal(n, x)


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_gradients_are_those_of_differences(neighbours, norm):
    rng, x, angle = setting(8, 16, seed=3)
    gain, grad, h = rng.standard_normal(16) if norm else None, rng.standard_normal(x.shape), 1e-6
    f = lambda x, gain: (O.rope_forward_real(x, angle, neighbours, norm, gain, 1e-3)[0] * grad).sum()
    dx, dg = O.rope_backward_real(x, angle, neighbours, norm, gain, 1e-3, grad)
    for _ in range(20):
        d = rng.standard_normal(x.shape)
        assert np.isclose((f(x + h * d, gain) - f(x - h * d, gain)) / (2 * h), (dx * d).sum(), rtol=1e-6, atol=1e-6)
        if norm:
            d = rng.standard_normal(16)
            assert np.isclose((f(x, gain + h * d) - f(x, gain - h * d)) / (2 * h), (dg * d).sum(), rtol=1e-6, atol=1e-6)


def test_key_weights_sum_to_the_queries_that_see_something():
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((9, 4, 8)), rng.standard_normal((6, 2, 8))
    assert np.allclose(O.key_weights_real(q, k, False, 0.3).sum(1), 18)
    assert np.allclose(O.key_weights_real(q, k, True, 0.3).sum(1), 12)          # the first three queries see nothing
    assert np.allclose(O.key_weights_real(q, k, True, 0.3, last=2).sum(1), 4)
    assert np.allclose(O.key_weights_real(q, k, True, 0.3, last=0), 0)


def test_eviction_keeps_what_its_order_says():
    w = [0.5, 0.0, np.nan, 2.0, 0.5, 0.0, 0.1]
    assert O.evict_choice(w, 3, 0, 0).tolist() == [0, 3, 4]
    assert O.evict_choice(w, 2, 0, 0).tolist() == [0, 3]             # equal weights: the lower index
    assert O.evict_choice(w, 3, 1, 1).tolist() == [0, 3, 6]
    assert O.evict_choice(w, 3, 2, 2).tolist() == [0, 1, 5]          # more stay than fit: by index
    assert O.evict_choice(w, 6, 0, 0).tolist() == [0, 1, 3, 4, 5, 6]
    assert O.evict_choice(w, 9, 0, 0).tolist() == list(range(7)) and O.evict_choice(w, 0, 3, 3).tolist() == []
    assert O.evict_choice([np.nan, np.inf, -np.inf, 1.0], 3, 0, 0).tolist() == [1, 2, 3]
