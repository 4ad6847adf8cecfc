"""Norms in place where a work-group takes several rows, ragged ones of several waves among them, whose last unit begins inside another wave's: results are those of calls with
outputs of their own, value by value."""
import pytest

from tests.test_rms_norm_gpu import TYPES

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def anr():
    from paper_2006_06762_amd import binding
    return binding


# more rows than the backward pass has at a time: 256 work-groups of one row from 577 threads on, at least as many rows by fewer
SIZES = [(7001, 99), (2900, 515), (1700, 1363), (1100, 2049), (1100, 4100), (900, 6149), (700, 8191), (530, 9001), (530, 16385)]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("T,C", SIZES)
def test_gradients(anr, t, T, C):
    t, g = TYPES[t], torch.Generator(device="cuda").manual_seed(T)
    ins = [torch.randn(T, C, generator=g, device="cuda").to(t) for _ in range(3)]
    gamma, rstd = torch.randn(C, generator=g, device="cuda").to(t), torch.rand(T, generator=g, device="cuda") + 0.5
    dx, dgamma = torch.full_like(ins[0], float("nan")), torch.full_like(gamma, float("nan"))
    anr.rms_norm_backward(ins[0], ins[1], gamma, rstd, dx, dgamma, ins[2])
    for which, name in enumerate(("dy", "x", "dh")):
        dy, x, dh = (v.clone() for v in ins)
        dg = torch.full_like(gamma, float("nan"))
        anr.rms_norm_backward(dy, x, gamma, rstd, (dy, x, dh)[which], dg, dh)
        assert torch.equal((dy, x, dh)[which], dx) and torch.equal(dg, dgamma), name


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("T,C", SIZES)
def test_norms(anr, t, T, C):
    t, g = TYPES[t], torch.Generator(device="cuda").manual_seed(C)
    x, res = (torch.randn(T, C, generator=g, device="cuda").to(t) for _ in range(2))
    gamma = torch.randn(C, generator=g, device="cuda").to(t)
    y, h, q, scale = torch.empty_like(x), torch.empty_like(x), torch.empty(T, C, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    anr.rms_norm(x, y, gamma, 1e-6, res, h)
    anr.rms_norm_q8(x, q, scale, gamma, 1e-6, res)
    for over_x in (True, False):
        a, b = x.clone(), res.clone()
        anr.rms_norm(a, b if over_x else a, gamma, 1e-6, b, a if over_x else b)
        assert torch.equal(a if over_x else b, h) and torch.equal(b if over_x else a, y)
        a, b, q2, scale2 = x.clone(), res.clone(), torch.empty_like(q), torch.empty_like(scale)
        anr.rms_norm_q8(a, q2, scale2, gamma, 1e-6, b, a if over_x else b)
        assert torch.equal(a if over_x else b, h) and torch.equal(q2, q) and torch.equal(scale2, scale)
