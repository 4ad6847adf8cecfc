"""Group norm at the sizes and values where its division of the work and its sums can go wrong, against the definition in 64 bits."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from test_blocks_gpu import HALF, O, TYPES, U, anr, dev, host, images, nans, norm_case, rng, within  # noqa: E402,F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t,shape,spare", [("bf16", (2, 120, 40, 41, 3), 0), ("bf16", (1, 120, 70, 41, 24), 0), ("f32", (2, 51, 30, 31, 3), 0), ("f32", (1, 95, 60, 31, 19), 0),
                                           ("f16", (2, 320, 40, 20, 32), 1), ("f32", (2, 192, 60, 31, 32), 1), ("bf16", (1, 448, 33, 21, 32), 1), ("f32", (1, 200, 90, 31, 40), 0),
                                           ("f32", (3, 48, 20, 20, 4), 0), ("bf16", (2, 144, 20, 20, 6), 0)])
def test_a_last_chunk_of_fewer_channels(anr, t, shape, spare):
    """Whose work-groups have more rows of threads than those of a full chunk."""
    N, C, H, W, groups = shape
    norm_case(anr, 80, N, C, H, W, groups, "silu", TYPES[t], spare=spare)
