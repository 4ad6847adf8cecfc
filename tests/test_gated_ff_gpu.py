"""The gated feed-forward block where it changes from one way to another."""
import pytest

torch = pytest.importorskip("torch")
from test_blocks_gpu import TYPES, anr, ff_case  # noqa: E402,F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("T,C,F", [(17, 1024, 9000), (32, 1024, 5632), (33, 1024, 5632), (40, 1025, 3999), (64, 768, 2816), (64, 1024, 4096), (64, 520, 7001)])
def test_up_to_64_tokens_of_wide_layers(anr, t, T, C, F):
    """Both sides of the line between the kernel of few tokens and tiles."""
    ff_case(anr, 90, T, C, F, "silu", TYPES[t], backward=False)
    ff_case(anr, 91, T, C, F, "gelu", TYPES[t], save=False, backward=False)
