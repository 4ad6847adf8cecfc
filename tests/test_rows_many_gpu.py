"""More rows than a launch has work-groups: those beyond are taken in turn, and are what they are in a call of their own."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def anr():
    from paper_2006_06762_amd import binding
    return binding


def edges(T):
    """Rows of the first turn, of its end and of the second."""
    return torch.tensor([0, 1, 1000, (1 << 20) - 1, 1 << 20, (1 << 20) + 1, T - 2, T - 1], device="cuda")


@pytest.mark.parametrize("C", [2048, 2051])
def test_rows_in_turn(anr, C):
    T = (1 << 20) + 9
    x = torch.empty(T, C, dtype=torch.bfloat16, device="cuda").normal_()
    y, q, scale, rstd = torch.empty_like(x), torch.empty(T, C, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    gamma = torch.randn(C, device="cuda").bfloat16()
    at = edges(T)
    part = x[at].contiguous()
    n = len(at)
    py, pq, pscale, prstd = torch.empty_like(part), torch.empty(n, C, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")

    def same(*pairs):
        for whole, own in pairs:
            assert torch.equal(whole[at], own)

    anr.rms_norm(x, y, gamma, 1e-6, rstd=rstd)
    anr.rms_norm(part, py, gamma, 1e-6, rstd=prstd)
    # (a row's sum goes by the threads that have it, few rows have one unit a thread, many two: each is within 32 u of the definition, u = 2^-24, and y's are then the same or neighbours)
    assert torch.allclose(rstd[at], prstd, rtol=64 * 2.0 ** -24, atol=0)
    assert bool((rstd > 0).all()) and bool(((y[at].float() - py.float()).abs() <= py.float().abs() * 2.0 ** -7).all())
    anr.rms_norm_q8(x, q, scale, gamma, 1e-6)
    anr.rms_norm_q8(part, pq, pscale, gamma, 1e-6)
    assert torch.allclose(scale[at], pscale, rtol=64 * 2.0 ** -24, atol=0)
    same((q, pq))
    q.zero_()
    scale.zero_()
    anr.quantize_rows(x, q, scale, anr.ANR_ACT_SILU)
    anr.quantize_rows(part, pq, pscale, anr.ANR_ACT_SILU)
    same((q, pq), (scale, pscale))
    assert bool((scale > 0).all()) and bool((q.abs().amax(1) == 127).all())
    y.zero_()
    anr.dequantize_rows(q, scale, y)
    anr.dequantize_rows(pq, pscale, py)
    same((y, py))
    # in place, over the rows of both turns
    z = x.clone()
    anr.rms_norm(x, y, gamma, 1e-6)
    anr.rms_norm(z, z, gamma, 1e-6)
    assert torch.equal(z, y)
