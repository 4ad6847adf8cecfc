"""Products of 8-bit integers: every kernel that a call can run, by the products that choose it (tests/test_gemm_i8_plan_cpu.py holds the shapes to their kernels).

Bounds as in tests/test_gemm_i8_gpu.py: the sum, exact in 64 bits, takes three roundings of 2^-24, one with a bias, and that to its type."""
import pytest

from tests.test_rms_norm_gpu import HALF, TINY, TYPES, U, untouched

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

# (edges of the tile, its buffers, whether work-groups share k): M, N, k.  Each product is run with N, whole lines of results, and N + 3, with k, whose rows start at whole words, and with
# k + 1, whose rows start at any byte.  k ends inside a chunk.
TILED = {
    (256, 256, 2, False): (700, 11328, 260), (256, 256, 2, True): (133, 8384, 18488),
    (128, 128, 2, False): (330, 11072, 260), (128, 128, 2, True): (65, 11072, 8284),
    (128, 128, 3, False): (140, 11072, 1300), (128, 128, 3, True): (65, 4160, 8548),
    (64, 128, 3, False): (70, 8320, 260), (64, 128, 3, True): (65, 1664, 6692),
    (64, 64, 3, False): (100, 704, 260), (64, 64, 3, True): (70, 320, 3000),
    (64, 64, 4, False): (70, 704, 1500), (64, 64, 4, True): (65, 2112, 4508),
}
# (blocks of sixteen rows, waves): M, N, k of the kernels for few rows, run alike.
ROWS = {
    (1, 4): (9, 704, 516), (1, 8): (9, 704, 2300), (1, 16): (9, 704, 8700), (2, 4): (20, 704, 516), (2, 8): (20, 704, 2300),
    (3, 4): (40, 704, 516), (4, 4): (60, 704, 516),
}


@pytest.fixture(scope="module")
def anr():
    from paper_2006_06762_amd import binding
    return binding


def whole(g, rows, k, shift=0):
    """[rows,k] in a storage with 77 in front of and behind it."""
    store = torch.full((rows * k + 64,), 77, dtype=torch.int8, device="cuda")
    view = store[16 + shift:16 + shift + rows * k].view(rows, k)
    view.copy_(torch.randint(-128, 128, (rows, k), generator=g, device="cuda", dtype=torch.int8))
    return view


def check(got, a, w, sa, sw, bias, t):
    sums = a.double() @ w.double().t().contiguous()
    v = sums * sa.double()[:, None] * sw.double()
    want = v if bias is None else v + bias.double()
    bound = 3.01 * U * v.abs() + U * want.abs() * (bias is not None)
    over = (got.double() - want).abs() - (bound + HALF[t] * (want.abs() + bound) + TINY[t])
    assert not torch.isnan(got).any() and float(over.max()) <= 0, int(over.argmax())


def product(anr, t, M, N, K, bias):
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    a, w = whole(g, M, K, K % 2), whole(g, N, K, 2 * (K % 2))
    rand = lambda n, hi: torch.rand(n, generator=g, device="cuda") * hi + hi / 16  # noqa: E731
    sa, sw = rand(M, 0.01), rand(N, 0.001)
    b = torch.randn(N, generator=g, device="cuda").to(t) if bias else None
    store = torch.full((M * N + 256,), float("nan"), dtype=t, device="cuda")
    d = store[128:128 + M * N].view(M, N)
    assert d.data_ptr() % 128 == 0
    anr.gemm_i8(a, w, sa, sw, d, b)
    assert untouched(d) and untouched(a) and untouched(w)
    check(d, a, w, sa, sw, b, t)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("kernel", [*TILED, *ROWS], ids=str)
def test_every_kernel(anr, t, kernel):
    M, N, K = (TILED if kernel in TILED else ROWS)[kernel]
    for n in (N, N + 3):
        for k in (K, K + 1):
            print(kernel, t, M, n, k, flush=True)
            product(anr, TYPES[t], M, n, k, bias=n != N)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("M", [260, 40, 3])
def test_longest_rows_between(anr, t, M):
    """Rows of operands far apart: the offsets in a tile are the largest, and those of its bytes all four."""
    g = torch.Generator(device="cuda").manual_seed(M)
    for ld in (300001, 300000):
        a, w = (torch.randint(-128, 128, (s, ld), generator=g, device="cuda", dtype=torch.int8) for s in (M, 140))
        a, w = a[:, 4:1005], w[:, 77776:78777]
        sa, sw = torch.rand(M, generator=g, device="cuda") * 0.01, torch.rand(140, generator=g, device="cuda") * 0.001
        d = torch.full((M, 140), float("nan"), dtype=TYPES[t], device="cuda")
        anr.gemm_i8(a, w, sa, sw, d)
        check(d, a, w, sa, sw, None, TYPES[t])
