"""What the block operators ask for as a workspace."""
import pytest

pytest.importorskip("torch")
from paper_2006_06762_amd import binding as B  # noqa: E402


def need(T, C, F, op=B.ANR_OP_GATED_FF, **kw):
    return B.workspace_size(op, B.GatedFfDesc(T=T, C=C, F=F, act=B.ANR_ACT_SILU, dtype=B.ANR_F32, **kw))


def test_a_float32_forward_call_keeps_its_hidden_values_once():
    """Gate and up are in the workspace only where they are products of their own: operands beyond what one launch for both takes."""
    for T, C, F in ((100, 64, 96), (8192, 4096, 11264), (3, 4096, 11264), (1300, 2048, 640)):
        assert T * F * 4 <= need(T, C, F) < T * F * 4 * 1.01 + 8 * T * C * 4, (T, C, F)
    far = 1 << 21
    for kw in ({"ldx": far}, {"ldw": far}):
        assert need(1000, 64, 1000, **kw) >= 3 * 1000 * 1000 * 4
    assert need((1 << 22) - 1, 136, 16) >= 3 * ((1 << 22) - 1) * 16 * 4
