"""Pins of the float64 oracle of the linear products, LayerNorm and dropout: the generator's published
vectors, gradients against central differences."""
import numpy as np
import pytest

from oracle import train as ot


@pytest.mark.parametrize("rounds,counter,key,want", [
    # the known-answer vectors published with the generator's paper
    (10, (0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    (7, (0, 0, 0, 0), (0, 0), (0x5F6FB709, 0x0D893F64, 0x4F121F81, 0x4F730A48)),
    (7, (0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x5207DDC2, 0x45165E59, 0x4D8EE751, 0x8C52F662)),
])
def test_generator_vectors(rounds, counter, key, want):
    assert tuple(int(v) for v in ot.philox4x32(counter, key, rounds)) == want


def test_keep_rate_and_independence():
    n = 1 << 20
    for p in (0.1, 0.5, 0.9):
        k = ot.keep(n, p, seed=7)
        q = 1.0 - ot.threshold(p) / 65536.0
        assert abs(k.mean() - q) < 5 * np.sqrt(q * (1 - q) / n)  # five standard deviations
    a, b = ot.keep(n, 0.5, seed=7), ot.keep(n, 0.5, seed=7, offset=1)
    assert abs((a == b).mean() - 0.5) < 5 * 0.5 / np.sqrt(n)
    assert (ot.keep(n, 0.5, 7, 2, 3) == ot.keep(n, 0.5, 7, 5)).all()
    assert (ot.keep(64, 0.5, 7, 2 ** 64 - 1, 1) == ot.keep(64, 0.5, 7, 0)).all()


def _differences(f, args, i, rng, step=1e-6):
    """d f / d args[i] along a random direction."""
    d = rng.standard_normal(args[i].shape)
    up, down = list(args), list(args)
    up[i], down[i] = args[i] + step * d, args[i] - step * d
    return (f(*up) - f(*down)) / (2 * step), d


@pytest.mark.parametrize("activation", ["none", "relu", "gelu"])
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_linear_gradients_are_differences(activation, p):
    rng = np.random.default_rng(3)
    x, w, b = rng.standard_normal((7, 5)), rng.standard_normal((5, 11)), rng.standard_normal(11)
    g = rng.standard_normal((7, 11))
    r = dict(p=p, seed=9, offset=4) if p else {}
    f = lambda *a: float((ot.linear(*a, activation, **r)[0] * g).sum())  # noqa: E731
    pre = ot.linear(x, w, b, activation)[1]
    grads = ot.linear_backward(g, x, w, pre, activation, **r)
    for i in range(3):
        num, d = _differences(f, (x, w, b), i, rng)
        assert abs(num - (grads[i] * d).sum()) < 1e-6 * max(1.0, abs(num))


def test_layer_norm_gradients_are_differences():
    rng = np.random.default_rng(4)
    v, ga, be = rng.standard_normal((6, 13)) + 3.0, rng.standard_normal(13), rng.standard_normal(13)
    g = rng.standard_normal(v.shape)
    f = lambda *a: float((ot.layer_norm(*a, 1e-6) * g).sum())  # noqa: E731
    grads = ot.layer_norm_backward(g, v, ga, 1e-6)
    for i in range(3):
        num, d = _differences(f, (v, ga, be), i, rng)
        assert abs(num - (grads[i] * d).sum()) < 1e-6 * max(1.0, abs(num))
