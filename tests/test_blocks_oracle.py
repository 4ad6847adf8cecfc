"""The definitions of oracle/blocks.py against closed forms and differences."""
import math

import numpy as np
import pytest

from oracle import blocks as O

ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")


def rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


def slope_of(f, x, step=1e-5):
    """Central differences of a scalar function of an array."""
    out = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        a, b = x.copy(), x.copy()
        a[i] += step
        b[i] -= step
        out[i] = (f(a) - f(b)) / (2 * step)
    return out


@pytest.mark.parametrize("name", ACTS)
def test_slopes_are_those_of_the_activations(name):
    z = np.array([-9.3, -2.0, -0.7, -1e-3, 2e-3, 0.4, 1.0, 3.3, 12.0])
    a, slope = O.act(name, z)
    assert np.allclose(slope, (O.act(name, z + 1e-6)[0] - O.act(name, z - 1e-6)[0]) / 2e-6, atol=1e-8)
    assert np.allclose(O.act(name, np.array([40.0]))[0], 40.0) and abs(O.act(name, np.array([0.0]))[0][0]) == 0
    assert O.act("silu", np.array([1.0]))[0][0] == pytest.approx(1 / (1 + math.exp(-1)))
    assert O.act("gelu", np.array([1.0]))[0][0] == pytest.approx(0.8413447460685429)


def test_group_norm_closed_forms():
    x = rng(1).normal(size=(3, 12, 4, 5)) * 3 + 7
    one, zero = np.ones(12), np.zeros(12)
    y, mean, rstd, _ = O.group_norm(x, 4, one, zero, 0.0, "none")
    v = y.reshape(3, 4, -1)
    assert np.allclose(v.mean(2), 0, atol=1e-12) and np.allclose((v ** 2).mean(2), 1)
    assert np.allclose(mean[1, 2], x[1, 6:9].mean()) and np.allclose(rstd[1, 2], 1 / x[1, 6:9].std())
    g, b = rng(2).normal(size=12), rng(3).normal(size=12)
    z = O.group_norm(x, 4, g, b, 0.0, "none")[0]
    assert np.allclose(z, y * g[:, None, None] + b[:, None, None])
    assert np.allclose(O.group_norm(x * 5 + 2, 4, g, b, 0.0, "silu")[0], O.act("silu", z)[0])


@pytest.mark.parametrize("name", ACTS)
def test_group_norm_gradients_are_differences(name):
    r = rng(4)
    x, dy, g, b = r.normal(size=(2, 6, 3)), r.normal(size=(2, 6, 3)), r.normal(size=6) + 1, r.normal(size=6)
    loss = lambda x, g, b: float((O.group_norm(x, 2, g, b, 1e-3, name)[0] * dy).sum())  # noqa: E731
    _, mean, rstd, _ = O.group_norm(x, 2, g, b, 1e-3, name)
    dx, dg, db = O.group_norm_backward(dy, x, 2, g, b, mean, rstd, name)[:3]
    assert np.allclose(dx, slope_of(lambda v: loss(v, g, b), x), atol=1e-7)
    assert np.allclose(dg, slope_of(lambda v: loss(x, v, b), g), atol=1e-7)
    assert np.allclose(db, slope_of(lambda v: loss(x, g, v), b), atol=1e-7)


@pytest.mark.parametrize("pairing", ["halves", "adjacent", "section_halves"])
def test_rotary_turns_pairs(pairing):
    r = rng(5)
    x, sections, freq = r.normal(size=(2, 3, 2, 14)), (2, 1, 3), r.uniform(0.1, 1, size=6)
    pos = r.integers(0, 50, size=(3, 2, 3))
    y = O.rotary(x, pos, freq, sections, pairing, False)
    assert np.allclose(O.rotary(y, pos, freq, sections, pairing, True), x)
    assert np.array_equal(y[..., 12:], x[..., 12:])
    first, second = O.rotary_pairs(sections, pairing)
    assert sorted([*first, *second]) == list(range(12))
    z, w = x[..., first] + 1j * x[..., second], y[..., first] + 1j * y[..., second]
    axis = np.array([0, 0, 1, 2, 2, 2])
    assert np.allclose(w / z, np.exp(1j * pos[axis].transpose(1, 2, 0) * freq)[:, :, None])
    # scores depend on differences of positions only
    q, k = r.normal(size=(2, 1, 3, 1, 14))
    turned = lambda shift: (O.rotary(q, pos[:, :1] + shift, freq, sections, pairing, False) * O.rotary(k, pos[:, :1] + shift + 3, freq, sections, pairing, False)).sum()  # noqa: E731
    assert turned(0) == pytest.approx(turned(11))
    if pairing == "section_halves":
        assert list(first) == [0, 1, 4, 6, 7, 8] and list(second) == [2, 3, 5, 9, 10, 11]


@pytest.mark.parametrize("name", ACTS)
def test_gated_ff_gradients_are_differences(name):
    r = rng(6)
    x, wg, wu, wd, dy = r.normal(size=(3, 4)), r.normal(size=(5, 4)), r.normal(size=(5, 4)), r.normal(size=(4, 5)), r.normal(size=(3, 4))
    loss = lambda *a: float((O.gated_ff(*a, name)[0] * dy).sum())  # noqa: E731
    _, gate, up = O.gated_ff(x, wg, wu, wd, name)
    got = O.gated_ff_backward(dy, x, wg, wu, wd, gate, up, name)
    args = [x, wg, wu, wd]
    for i, g in enumerate(got):
        want = slope_of(lambda v: loss(*args[:i], v, *args[i + 1:]), args[i])
        assert np.allclose(g, want, atol=1e-6)


def test_gated_ff_closed_form():
    # one channel, one hidden unit: y = act(a x) b x c
    y, gate, up = O.gated_ff(np.array([[2.0]]), np.array([[1.5]]), np.array([[-0.5]]), np.array([[4.0]]), "relu")
    assert (gate[0, 0], up[0, 0], y[0, 0]) == (3.0, -1.0, -12.0)
