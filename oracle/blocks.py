"""Definitions of the operators of a transformer block in 64 bits, on numpy arrays: group norm with an activation, rotary
positions with several axes, the gated feed-forward block, and their gradients.  Test infrastructure; shares no code with
the GPU path."""
import math

import numpy as np

_erf = np.vectorize(math.erf, otypes=[float])


def _sigmoid(z):
    return np.where(z >= 0, 1 / (1 + np.exp(-np.abs(z))), np.exp(-np.abs(z)) / (1 + np.exp(-np.abs(z))))


def act(name, z):
    """(act(z), act'(z)) for "none", "relu", "silu", "gelu", "gelu_tanh"."""
    z = np.asarray(z, np.float64)
    if name == "relu":
        return np.maximum(z, 0), (z > 0).astype(float)
    if name == "silu":
        s = _sigmoid(z)
        return z * s, s + z * s * (1 - s)
    if name == "gelu":
        phi = 0.5 * (1 + _erf(z / math.sqrt(2)))
        return z * phi, phi + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        a, b = math.sqrt(2 / math.pi), 0.044715
        t = np.tanh(a * (z + b * z ** 3))
        return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * a * (1 + 3 * b * z * z)
    assert name == "none"
    return z.copy(), np.ones_like(z)


def group_norm(x, groups, gamma, beta, eps, activation):
    """x [N,C,...]; (y, mean [N,G], rstd [N,G], z) with z what the activation takes."""
    N, C = x.shape[:2]
    v = x.reshape(N, groups, -1)
    mean = v.mean(2)
    rstd = 1 / np.sqrt(((v - mean[:, :, None]) ** 2).mean(2) + eps)
    hat = ((v - mean[:, :, None]) * rstd[:, :, None]).reshape(x.shape)
    per = (1, C) + (1,) * (x.ndim - 2)
    z = hat * gamma.reshape(per) + beta.reshape(per)
    return act(activation, z)[0], mean, rstd, z


def group_norm_backward(dy, x, groups, gamma, beta, mean, rstd, activation):
    """(dx, dgamma, dbeta, and for error bounds: dz, hat, the group's means of |dz gamma| and |dz gamma hat| at each element)."""
    N, C = x.shape[:2]
    per, rest = (1, C) + (1,) * (x.ndim - 2), (0,) + tuple(range(2, x.ndim))
    of_group = lambda s: np.broadcast_to(s[:, :, None], (N, groups, x[0].size // groups)).reshape(x.shape)  # noqa: E731
    hat = (x - of_group(mean)) * of_group(rstd)
    dz = dy * act(activation, hat * gamma.reshape(per) + beta.reshape(per))[1]
    d = dz * gamma.reshape(per)
    means = lambda v: of_group(v.reshape(N, groups, -1).mean(2))  # noqa: E731
    dx = of_group(rstd) * (d - means(d) - hat * means(d * hat))
    return dx, (dz * hat).sum(rest), dz.sum(rest), dz, hat, means(np.abs(d)), means(np.abs(d * hat))


def rotary_pairs(sections, pairing):
    """(first, second): the two dimensions of each pair."""
    n = sum(sections)
    if pairing == "adjacent":
        return np.arange(n) * 2, np.arange(n) * 2 + 1
    if pairing == "halves":
        return np.arange(n), np.arange(n) + n
    first, second, block = [], [], 0
    for s in sections:
        first += range(block, block + s)
        second += range(block + s, block + 2 * s)
        block += 2 * s
    return np.array(first, int), np.array(second, int)


def rotary(x, positions, inv_freq, sections, pairing, inverse):
    """x [B,S,H,D], positions [axes,B,S], inv_freq [pairs]."""
    axis = np.repeat(np.arange(len(sections)), sections)
    angle = np.moveaxis(positions[axis].astype(np.float64), 0, -1) * inv_freq.astype(np.float64)
    c, s = np.cos(angle)[:, :, None], np.sin(angle)[:, :, None] * (-1 if inverse else 1)
    first, second = rotary_pairs(sections, pairing)
    y = x.copy()
    y[..., first] = x[..., first] * c - x[..., second] * s
    y[..., second] = x[..., first] * s + x[..., second] * c
    return y


def gated_ff(x, w_gate, w_up, w_down, activation):
    """(y, gate, up)."""
    gate, up = x @ w_gate.T, x @ w_up.T
    return (act(activation, gate)[0] * up) @ w_down.T, gate, up


def gated_ff_backward(dy, x, w_gate, w_up, w_down, gate, up, activation):
    """(dx, dw_gate, dw_up, dw_down)."""
    a, slope = act(activation, gate)
    dh = dy @ w_down
    dg, du = dh * up * slope, dh * a
    return dg @ w_gate + du @ w_up, dg.T @ x, du.T @ x, dy.T @ (a * up)
