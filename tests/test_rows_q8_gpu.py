"""Rows of values in 8 bits with a scale each, and back, against their definitions in 64 bits (oracle/blocks.py).

Activations are evaluated to 64 u of 1 + |z|, u = 2^-24 (the quick exponential's argument is rounded, 1.5 |z| u, and what follows are a few
roundings; |z| stays below 20 here), the product with up once more.  The scale is a 127th of the largest value, rounded; q the nearest whole number
to the value times the step's inverse (three roundings)."""
import numpy as np
import pytest

from oracle import blocks as O
from tests.test_rms_norm_gpu import HALF, TINY, TYPES, U, host, matrix, rng, untouched

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")


@pytest.fixture(scope="module")
def anr():
    from paper_2006_06762_amd import binding
    return binding


def case(anr, seed, T, C, t, act="none", gated=False, spare=0, shift=0):
    r = rng(seed)
    x = matrix(r.normal(size=(T, C)) * r.uniform(0.1, 3, size=(T, 1)), t, spare, shift)
    up = matrix(r.normal(size=(T, C)), t, spare, shift) if gated else None
    q, scale = matrix(np.zeros((T, C)), torch.int8, spare, shift), torch.full((T,), float("nan"), device="cuda")
    got = anr.quantize_rows(x, q, scale, getattr(anr, "ANR_ACT_" + act.upper()), up)
    assert got[0] is q and got[1] is scale and untouched(q) and untouched(x)
    z = host(x)
    v, off = O.act(act, z)[0], (64 * U * (1 + np.abs(z))) * (act not in ("none", "relu"))
    if gated:
        v, off = v * host(up), off * np.abs(host(up))
    off = off + U * np.abs(v)
    steps, s = O.in_8_bits(v)
    es = off.max(1) / 127 + 2 * U * s
    assert np.all(np.abs(host(scale) - s) <= es)
    some = s > 0
    bound = 0.5 + ((off + 127 * es[:, None]) / np.where(some, s, 1)[:, None]) + 127 * 4 * U
    assert np.all(np.abs(host(q) - steps) <= bound)
    assert np.all(np.abs(host(q)).max(1) == 127 * some)
    # and back
    for kind in TYPES.values():
        y = matrix(np.full((T, C), np.nan), kind, spare, shift)
        assert anr.dequantize_rows(q, scale, y) is y and untouched(y)
        want = host(q) * host(scale)[:, None]
        assert np.all(np.abs(host(y) - want) <= HALF[torch.float32] * np.abs(want) + HALF[kind] * np.abs(want) * (1 + U) + TINY[kind])


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("C", [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 63, 64, 100, 515, 1001, 1363, 2048, 4096, 5632, 11264, 16384, 32768, 32769, 40000, 100003])
def test_widths(anr, t, C):
    for T in (1, 3) if C > 4096 else (1, 2, 37, 1030):
        print(t, T, C, flush=True)
        case(anr, 1, T, C, TYPES[t], "silu", True)
    case(anr, 2, 5, C, TYPES[t])


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("act", ACTS)
def test_activations(anr, t, act, gated):
    case(anr, 3, 21, 264, TYPES[t], act, gated)
    case(anr, 4, 2, 33000, TYPES[t], act, gated)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("spare,shift", [(8, 0), (3, 0), (0, 1), (5, 3), (16, 8)])
def test_strides(anr, t, spare, shift):
    for T, C in ((9, 40), (1025, 264), (2, 1363), (3, 6), (2, 32771)):
        case(anr, 5, T, C, TYPES[t], "gelu", True, spare, shift)


def test_halves_of_one_product(anr):
    """Gate and up side by side, as one product leaves them."""
    both = torch.randn(50, 2 * 96, device="cuda").bfloat16()
    q, scale, q2, scale2 = torch.empty(50, 96, dtype=torch.int8, device="cuda"), torch.empty(50, device="cuda"), torch.empty(50, 96, dtype=torch.int8, device="cuda"), torch.empty(50, device="cuda")
    anr.quantize_rows(both[:, :96], q, scale, anr.ANR_ACT_SILU, both[:, 96:])
    anr.quantize_rows(both[:, :96].contiguous(), q2, scale2, anr.ANR_ACT_SILU, both[:, 96:].contiguous())
    assert torch.equal(q, q2) and torch.equal(scale, scale2)


def test_ties_go_to_even(anr):
    x = torch.tensor([[127.0, 0.5, 1.5, 2.5, -0.5, -1.5, -2.5, 126.5]], device="cuda")
    q, scale = torch.empty(1, 8, dtype=torch.int8, device="cuda"), torch.empty(1, device="cuda")
    anr.quantize_rows(x, q, scale)
    assert q.tolist() == [[127, 0, 2, 2, 0, -2, -2, 126]] and scale.item() == 1


@pytest.mark.parametrize("C", [6, 300, 33001])
def test_special_values(anr, C):
    x = torch.randn(9, C, device="cuda")
    x[1] = 0
    x[2, C - 1] = float("nan")
    x[3, 0] = float("inf")
    x[4] *= 1e-38
    x[5] *= 2.0 ** -140                         # below float32's normal range
    x[6] *= 1e37
    x[7, 1] = -float("inf")
    x[8] = -0.0
    q, scale, y = torch.empty(9, C, dtype=torch.int8, device="cuda"), torch.empty(9, device="cuda"), torch.empty(9, C, device="cuda")
    anr.quantize_rows(x, q, scale)
    anr.dequantize_rows(q, scale, y)
    for row in (0, 4, 5, 6):
        steps, s = O.in_8_bits(host(x[row:row + 1]))
        assert abs(float(scale[row]) - s[0]) <= 2 * U * s[0] + 2.0 ** -150
        assert np.all(np.abs(host(q[row:row + 1]) - steps) <= 0.5 + 127 * 4 * U)
    for row in (1, 8):
        assert (q[row] == 0).all() and scale[row] == 0 and (y[row] == 0).all()
    for row in (2, 3, 7):
        assert (q[row] == 0).all() and torch.isnan(scale[row]) and torch.isnan(y[row]).all()


def test_all_steps_come_back(anr):
    q = torch.arange(-128, 128, device="cuda").to(torch.int8).view(1, 256)
    for t in TYPES.values():
        y = torch.empty(1, 256, dtype=t, device="cuda")
        anr.dequantize_rows(q, torch.tensor([0.25], device="cuda"), y)
        assert torch.equal(y.float(), q.float() * 0.25)


def test_no_rows(anr):
    x, none = torch.empty(0, 64, device="cuda"), torch.empty(0, device="cuda")
    anr.quantize_rows(x, x.char(), none)
    anr.dequantize_rows(x.char(), none, x)
