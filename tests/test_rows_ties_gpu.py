"""Rows in 8 bits next to ties: q is v / scale to the nearest whole number, a half to the even one.

A row whose largest magnitude is 127 j 2^e (j odd, a few bits) has the scale j 2^e, which float32 holds, and (2 i + 1) j 2^(e - 1) lies i + 1/2
steps from zero, exactly: nothing is rounded up to there, and what is compared are whole numbers."""
import numpy as np
import pytest

from tests.test_rms_norm_gpu import TYPES, host, rng

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BITS = {"f32": 24, "f16": 11, "bf16": 8}


@pytest.fixture(scope="module")
def anr():
    from paper_2006_06762_amd import binding
    return binding


def halves(j, e, bits, C, gated=False):
    """[2,C] of 127 j 2^e and, in turn, what of (2 i + 1) j 2^(e - 1) and their negatives the type holds, and the steps; gated: without the factor j."""
    i = np.arange(127)
    i = i[(2 * i + 1) * (1 if gated else j) < 2 ** bits]
    odd = np.resize(np.concatenate([2 * i + 1, -(2 * i + 1)]), C - 1)
    steps = np.concatenate([[127.0], odd / 2])
    return np.stack([steps, -steps]) * (1 if gated else j) * 2.0 ** e, np.rint(np.stack([steps, -steps]))


def held(j, bits):
    while j % 2 == 0:
        j //= 2
    return 127 * j < 2 ** bits


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("C", [300, 4096, 33001])
def test_halves_of_a_step(anr, t, C):
    for j in range(1, 1000 if t == "f32" and C == 300 else 33, 2):
        if not held(j, BITS[t]):
            continue
        for e in (-9, 0, 3) if t == "f16" else (-140 if t == "f32" else -130, -100, -7, 0, 90, 110):
            if j * 127 * 2.0 ** e > (60000 if t == "f16" else 2.0 ** 127):
                continue
            v, want = halves(j, e, BITS[t], C)
            x = torch.from_numpy(v).to(TYPES[t]).cuda()
            assert np.array_equal(host(x), v)
            q, scale = torch.empty(2, C, dtype=torch.int8, device="cuda"), torch.empty(2, device="cuda")
            anr.quantize_rows(x, q, scale)
            assert (scale == j * 2.0 ** e).all()
            assert np.array_equal(host(q), want), (j, e, v[host(q) != want][:4] / (j * 2.0 ** e), host(q)[host(q) != want][:4])


@pytest.mark.parametrize("t", TYPES)
def test_halves_of_a_step_gated(anr, t):
    """The product with up is exact: nine bits by at most ten."""
    C = 264
    for j in range(1, 255, 2):
        if j >= 2 ** BITS[t]:
            continue
        v, want = halves(j, 0, BITS[t], C, gated=True)
        keep = np.abs(v).max() * j < 2 ** 15
        if not keep:
            continue
        x, up = torch.from_numpy(v).to(TYPES[t]).cuda(), torch.full((2, C), float(j), device="cuda").to(TYPES[t])
        q, scale = torch.empty(2, C, dtype=torch.int8, device="cuda"), torch.empty(2, device="cuda")
        anr.quantize_rows(x, q, scale, anr.ANR_ACT_NONE, up)
        assert (scale == j).all() and np.array_equal(host(q), want), j


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("C", [300, 4096])
def test_halves_of_a_step_of_a_norm(anr, t, C):
    """Whatever rstd is, the values are its multiples."""
    for j in range(1, 127, 2):
        if j >= 2 ** BITS[t]:
            continue
        v, want = halves(j, 0, BITS[t], C, gated=True)
        x, gamma = torch.from_numpy(v).to(TYPES[t]).cuda(), torch.full((C,), float(j), device="cuda").to(TYPES[t])
        q, scale = torch.empty(2, C, dtype=torch.int8, device="cuda"), torch.empty(2, device="cuda")
        anr.rms_norm_q8(x, q, scale, gamma, 1e-6)
        assert np.array_equal(host(q), want), j


def test_quotients_in_float32(anr):
    """q is the float32 quotient v / scale, rounded.  The kernels' quotient is off by less than 2^-44 before it is rounded to 24 bits; two numbers of 24 bits whose quotient
    lies so near the middle between two of 24 bits, at half a step, are one in 2^36."""
    for C, T in ((300, 500), (4096, 100), (33001, 10)):
        r = rng(C)
        v = (r.normal(size=(T, C)) * r.uniform(0.1, 3, size=(T, 1))).astype(np.float32)
        q, scale = torch.empty(T, C, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
        anr.quantize_rows(torch.from_numpy(v).cuda(), q, scale)
        s = scale.cpu().numpy()
        assert np.array_equal(s, np.abs(v).max(1) / np.float32(127))
        assert np.array_equal(q.cpu().numpy(), np.rint(v / s[:, None]))
