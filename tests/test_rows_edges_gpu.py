"""Rows in 8 bits whose scale is nothing, or no number: zeros, squares that all count as zeros, sums of squares beyond float32, scales below its smallest number; eps = 0
among them."""
import numpy as np
import pytest

from tests.test_rms_norm_gpu import TYPES, host

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def anr():
    from paper_2006_06762_amd import binding
    return binding


def normed(anr, x, gamma, eps, residual=None):
    y, q, scale = torch.empty_like(x), torch.full(x.shape, 55, dtype=torch.int8, device="cuda"), torch.full(x.shape[:1], 7.0, device="cuda")
    anr.rms_norm(x, y, gamma, eps, residual)
    anr.rms_norm_q8(x, q, scale, gamma, eps, residual)
    return y, q, scale


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("C", [5, 60, 300, 4096, 20000])
def test_rows_of_zeros(anr, t, C):
    """Scale and q are zero whatever eps is, in rows between others too, and where x and the residual cancel."""
    x = torch.randn(7, C, device="cuda").to(TYPES[t])
    res = torch.randn(7, C, device="cuda").to(TYPES[t])
    for row in (0, 3, 6):
        res[row] = -x[row]
    for eps in (0.0, 1e-30, 1e-6):
        _, q, scale = normed(anr, x, None, eps, res)
        for row in (0, 3, 6):
            assert scale[row] == 0 and (q[row] == 0).all()
        for row in (1, 2, 4, 5):
            assert scale[row] > 0 and q[row].abs().max() == 127
    _, q, scale = normed(anr, x, torch.zeros(C, dtype=TYPES[t], device="cuda"), 0.0)
    assert (scale == 0).all() and (q == 0).all()


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("C", [5, 300, 4096, 20000])
def test_squares_that_are_zeros(anr, t, C):
    """eps = 0 and squares below float32's range: rstd and y are infinite, which is a NaN for the scale and zeros for q."""
    x = (torch.randn(3, C, device="cuda").sign() * 2.0 ** -80).to(TYPES[t])
    y, q, scale = normed(anr, x, None, 0.0)
    assert torch.isinf(y).all() and torch.isnan(scale).all() and (q == 0).all()
    # (with an eps they are numbers: 2^-80 2^40)
    y, q, scale = normed(anr, x, None, 2.0 ** -80)
    assert (y.abs() == 2.0 ** -40).all() and (q.abs() == 127).all() and (scale == np.float32(2.0 ** -40) / np.float32(127)).all()


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_sums_beyond_float32(anr, t):
    """rstd and y are zeros then, and so are scale and q."""
    x = (torch.randn(3, 300, device="cuda").sign() * 2.0 ** 70).to(TYPES[t])
    y, q, scale = normed(anr, x, None, 1e-6)
    assert (y == 0).all() and (scale == 0).all() and (q == 0).all()


@pytest.mark.parametrize("C", [3, 300, 33001])
def test_scales_below_the_smallest_number(anr, C):
    """A 127th of 64 times the smallest number rounds to that, of 63 times to zero: q is zero there."""
    x = torch.full((4, C), 2.0 ** -149, dtype=torch.float64)
    x *= torch.tensor([63.0, 64.0, 1.0, 127.0], dtype=torch.float64)[:, None]
    x[:, 0] *= -1
    assert np.array_equal(host(x.float()), x.numpy())
    q, scale = torch.full((4, C), 55, dtype=torch.int8, device="cuda"), torch.empty(4, device="cuda")
    anr.quantize_rows(x.float().cuda(), q, scale)
    assert host(scale).tolist() == [0.0, 2.0 ** -149, 0.0, 2.0 ** -149]
    for row in (0, 2):
        assert (q[row] == 0).all()
    for row in (1, 3):
        assert q[row, 0] == -127 and (q[row, 1:] == 127).all()
    # the same by way of the norm, whose y is half of h here: squares that count as zeros and eps = 4
    q, scale = torch.full((4, 300), 55, dtype=torch.int8, device="cuda"), torch.empty(4, device="cuda")
    x = torch.full((4, 300), 2.0 ** -148, dtype=torch.float64) * torch.tensor([63.0, 64.0, 1.0, 127.0], dtype=torch.float64)[:, None]
    anr.rms_norm_q8(x.float().cuda(), q, scale, None, 4.0)
    assert host(scale).tolist() == [0.0, 2.0 ** -149, 0.0, 2.0 ** -149]
    assert [int(q[row, 0]) for row in range(4)] == [0, 127, 0, 127]
