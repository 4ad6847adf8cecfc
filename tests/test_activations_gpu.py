"""The activations where their values are small: relative to themselves, through a feed-forward block whose weights are units."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
from test_blocks_gpu import HALF, TINY, TYPES, U, anr, host  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def through_a_block(anr, z, t, act, scale):
    """act(z) and act'(z) by a block of elements of t: token i has z[i] in its first channel and 1 in its last one; gate is z, up the scale, a power of two that keeps
    small values from float16's denormals, and y what the activation gave, scaled and rounded once."""
    T, C = len(z), 16
    x = torch.zeros(T, C, dtype=t, device="cuda")
    x[:, 0], x[:, -1] = torch.from_numpy(z).to(t), 1
    assert np.array_equal(host(x[:, 0]), z)
    wg, wu, wd = torch.zeros(C, C, dtype=t, device="cuda"), torch.zeros(C, C, dtype=t, device="cuda"), torch.eye(C, dtype=t, device="cuda")
    wg[0, 0], wu[0, -1] = 1, scale
    y, gate, up, dx = (torch.empty_like(x) for _ in range(4))
    anr.gated_ff(x, wg, wu, wd, y, act, gate, up)
    assert np.array_equal(host(gate[:, 0]), z) and (up[:, 0] == scale).all()
    dy = torch.zeros_like(x)
    dy[:, 0] = 1
    anr.gated_ff_backward(dy, x, wg, wu, wd, gate, up, dx, act=act)
    return host(y[:, 0]) / scale, host(dx[:, 0]) / scale


def phi(z):
    return np.array([0.5 * math.erfc(-v / math.sqrt(2)) for v in z])


def check(name, z, got, want, bound, t, scale):
    over = np.abs(got - want) - (bound + HALF[t] * (np.abs(want) + bound) + TINY[t] / scale)
    at = int(np.argmax(over))
    assert over[at] <= 0, "%s(%g): got %r, want %r, bound %r" % (name, z[at], got[at], want[at], bound[at])


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("T", [9, 241])
def test_gelu_is_as_good_far_below_zero(anr, t, T):
    """Bounds relative to the value.  float32: 16 u for the polynomials and the roundings of their terms, and the exponential's argument, rounded, u z^2 / 2.  16 bits:
    the polynomial's 66 u, 16 u for the roundings of its terms, the hardware's exponential and reciprocal, and the argument's three roundings, 1.5 u z^2; the
    result's own rounding is a hundred times as much.  Two products with a unit, 1.1 u each, and with z.  The slope is the sum of two terms, each of which is as far
    off as itself."""
    t = TYPES[t]
    z = np.round(np.linspace(*((-6, 1) if t is torch.float16 else (-10, 5)), T) * 16) / 16
    scale = 2.0 ** 15 if t is torch.float16 else 1.0
    y, dx = through_a_block(anr, z, t, anr.ANR_ACT_GELU, scale)
    p, density = phi(z), np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    relative = 16 * U + z * z / 2 * U if t is torch.float32 else 82 * U + 1.5 * z * z * U
    check("gelu", z, y, z * p, (relative + 4 * U) * np.abs(z * p), t, scale)
    check("slope", z, dx, p + z * density, (relative + 4 * U) * (p + np.abs(z) * density), t, scale)


def test_gelu_slope_at_infinities_and_nan(anr):
    """1 above and 0 below, by way of the gate weights' gradient: token i has a one in channel i."""
    for t in TYPES.values():
        for T in (16, 200):
            x, dy, dw = torch.zeros(T, 16, dtype=t, device="cuda"), torch.zeros(T, 16, dtype=t, device="cuda"), torch.empty(16, 16, dtype=t, device="cuda")
            x[:16], dy[:, 0] = torch.eye(16, device="cuda"), 1
            eye, gate, up = torch.eye(16, dtype=t, device="cuda"), torch.zeros_like(x), torch.ones_like(x)
            gate[0, 0], gate[1, 0] = float("inf"), float("-inf")
            anr.gated_ff_backward(dy, x, eye, eye, eye, gate, up, None, dw, act=anr.ANR_ACT_GELU)
            assert dw[0].tolist() == [1.0, 0.0] + [0.5] * 14 and not dw[1:].any()
            gate[2, 0] = float("nan")
            anr.gated_ff_backward(dy, x, eye, eye, eye, gate, up, None, dw, act=anr.ANR_ACT_GELU)
            assert torch.isnan(dw[0]).all() and not dw[1:].any()
