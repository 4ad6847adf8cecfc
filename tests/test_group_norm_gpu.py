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


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("shape", [(1, 512, 7, 7, 32), (3, 64, 20, 20, 8), (1, 32, 128, 128, 4), (2, 30, 40, 31, 3), (24, 256, 28, 28, 32)])
@pytest.mark.parametrize("centre,first", [(0, 100), (0, -1000), (0, 60000), (500, 0), (500, -400)])
def test_statistics_do_not_depend_on_where_a_group_starts(anr, t, shape, centre, first):
    """The first value of each group far from the others, and all of them far from zero: maps that a work-group holds and others, vectors and single
    elements.  The mean is a sum in 64 bits, rounded once; the variance one too, or sums in 32 bits of at most 16, 64 and 6 squares after each other, each of a
    difference off by 2 u; its root halves that and adds three roundings: 64 u.  y: a difference and a product, and a float's last place of the two terms."""
    N, C, H, W, groups = shape
    r = rng(81)
    a = r.normal(size=(N, C, H, W)) + centre
    a[:, ::C // groups, 0, 0] += first
    x, gamma, beta = images(a, TYPES[t]), dev(r.normal(size=C) * 0.3 + 1, torch.float32), dev(r.normal(size=C) * 0.3, torch.float32)
    y, mean, rstd = torch.empty_like(x), nans(N, groups, dtype=torch.float32), nans(N, groups, dtype=torch.float32)
    anr.group_norm(x, groups, y, gamma, beta, 1e-5, anr.ANR_ACT_NONE, mean, rstd)
    b = host(beta).reshape(1, C, 1, 1)
    want, m64, r64, z = O.group_norm(host(x), groups, host(gamma), host(beta), 1e-5, "none")
    largest = np.abs(host(x).reshape(N, groups, -1)).max(2)
    within("mean", mean, m64, 2.0 ** -40 * largest, torch.float32)
    within("rstd", rstd, r64, 64 * U * r64, torch.float32)
    within("y", y, want, 70 * U * np.abs(z - b) + 4 * U * (np.abs(z) + np.abs(b)), TYPES[t])


def test_the_mean_of_values_that_cancel(anr):
    """Halves of opposite sign and a small rest: the sum is exact in 64 bits, the mean's distance from a value of 1000 four roundings off."""
    for edge in (12, 24, 100):
        x = torch.full((2, 64, edge, edge), 1000.0, device="cuda").contiguous(memory_format=torch.channels_last)
        x[:, :, ::2] = -1000.0
        x[:, :, 5, 7] += 2.0 ** -10
        mean, want = nans(2, 8, dtype=torch.float32), 2.0 ** -10 / edge ** 2
        anr.group_norm(x, 8, torch.empty_like(x), mean=mean)
        assert (np.abs(host(mean) - want) <= U * want + 4 * 1000 * 2.0 ** -53).all(), edge


def gradients_of_long_sums(anr, x, dy, groups, k):
    """dbeta, dgamma and dx of a norm without activation and parameters within k u of the sums of their terms' magnitudes, and what xhat's roundings make:
    a difference, to u of its terms, and a product.  In 64 bits on the GPU (the CPU takes minutes)."""
    N, C, S = x.shape
    mean, rstd = nans(N, groups, dtype=torch.float32), nans(N, groups, dtype=torch.float32)
    anr.group_norm(x, groups, torch.empty_like(x), mean=mean, rstd=rstd)
    dx, dgamma, dbeta = torch.empty_like(x), nans(C, dtype=torch.float32), nans(C, dtype=torch.float32)
    anr.group_norm_backward(dy, x, groups, None, None, mean, rstd, dx, dgamma, dbeta)
    of_group = lambda v: v.double().repeat_interleave(C // groups, 1)[:, :, None]  # noqa: E731
    means = lambda v: of_group(v.reshape(N, groups, -1).mean(2))  # noqa: E731
    m, s, d = of_group(mean), of_group(rstd), dy.double()
    hat = (x.double() - m) * s
    ehat = 4 * U * (hat.abs() + (x.double().abs() + m.abs()) * s)
    half = HALF[x.dtype]

    def close(name, got, want, bound, half):
        over = ((got.double() - want).abs() - bound - half * (want.abs() + bound)).max().item()
        assert over <= 0, "%s: %g over the bound" % (name, over)

    close("dbeta", dbeta, d.sum((0, 2)), k * U * d.abs().sum((0, 2)), U)
    close("dgamma", dgamma, (d * hat).sum((0, 2)), k * U * (d * hat).abs().sum((0, 2)) + (d.abs() * ehat).sum((0, 2)), U)
    dhat = means((d * hat).abs())
    close("dx", dx, s * (d - means(d) - hat * means(d * hat)), s * (k * U * (d.abs() + means(d.abs()) + hat.abs() * dhat) + ehat * dhat + hat.abs() * means(d.abs() * ehat)), half)


@pytest.mark.parametrize("t,C,S", [("f32", 3, 1 << 24), ("f32", 4, 1 << 23), ("bf16", 8, 1 << 23), ("f16", 30, 1 << 20)])
def test_gradients_of_one_large_map(anr, t, C, S):
    """A gradient that is the same everywhere, of no whole number: sums of 32 in 32 bits, of those in 64, rounded, of at most eight slabs a lane and six joins, and
    four roundings of the terms: 50 u."""
    x = torch.randn(1, S, C, device="cuda").to(TYPES[t]).transpose(1, 2)
    gradients_of_long_sums(anr, x, torch.full_like(x, 0.7), 1, 50)
    torch.cuda.empty_cache()


@pytest.mark.parametrize("t,C", [("f32", 3), ("f32", 4), ("bf16", 8), ("f16", 5)])
def test_gradients_of_the_most_images(anr, t, C):
    """The parameters' sums over 65534 images of two pixels, 50 u as above."""
    x = torch.randn(65534, 2, C, device="cuda").to(TYPES[t]).transpose(1, 2)
    gradients_of_long_sums(anr, x, torch.full_like(x, 0.7), 1, 50)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("shape", [(1, 8192, 2, 1, 1), (2, 8192, 9, 5, 1), (1, 8184, 3, 1, 1), (1, 8191, 3, 2, 1)])
def test_the_widest_groups(anr, t, shape):
    """Whose sums take all of a CU's shared memory."""
    N, C, H, W, groups = shape
    norm_case(anr, 82, N, C, H, W, groups, "silu", TYPES[t])


@pytest.mark.parametrize("shape", [(16, 256, 24, 24, 32), (16, 256, 28, 28, 32), (4, 1024, 32, 32, 32), (16, 320, 23, 29, 32), (8, 512, 40, 40, 64)])
def test_float32_maps_held_by_half_the_work_groups(anr, shape):
    N, C, H, W, groups = shape
    norm_case(anr, 83, N, C, H, W, groups, "silu", torch.float32)


@pytest.mark.parametrize("t,shape", [("bf16", (1, 64, 300, 400, 8)), ("f32", (1, 64, 280, 330, 4)), ("f32", (2, 32, 250, 300, 32)), ("f16", (1, 5, 500, 401, 5))])
def test_as_many_slabs_as_are_joined(anr, t, shape):
    """One image, or two, of one or two chunks."""
    N, C, H, W, groups = shape
    norm_case(anr, 84, N, C, H, W, groups, "none", TYPES[t])
