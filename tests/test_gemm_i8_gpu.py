"""Products of 8-bit integers with scales against sums in whole numbers.

u = 2^-24.  The sum is exact; a result is it rounded to 24 bits, times two scales and with the bias added, a rounding each, and that to its type: three
roundings of the product, one of the sum with the bias."""
import numpy as np
import pytest

from tests.test_rms_norm_gpu import TYPES, U, host, matrix, rng, untouched, within

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def anr():
    from paper_2006_06762_amd import binding
    return binding


def case(anr, seed, M, N, K, t, bias=None, scales=True, spare=0, shift=0, extreme=False, spare_d=None):
    r = rng(seed)
    whole = (lambda *s: r.choice([-128, 127], size=s)) if extreme else (lambda *s: r.integers(-128, 128, size=s))  # noqa: E731
    a, w = matrix(whole(M, K), torch.int8, spare, shift), matrix(whole(N, K), torch.int8, spare, shift)
    f = lambda v: torch.from_numpy(v.astype(np.float32)).cuda()  # noqa: E731
    sa, sw = (f(r.uniform(0.001, 0.02, size=M)), f(r.uniform(0.0001, 0.002, size=N))) if scales else (None, None)
    b = torch.from_numpy(r.normal(size=N)).to(bias).cuda() if bias else None
    d = matrix(np.full((M, N), np.nan), t, spare if spare_d is None else spare_d, shift)
    assert anr.gemm_i8(a, w, sa, sw, d, b) is d
    assert untouched(d) and untouched(a) and untouched(w)
    sums = a.cpu().double().numpy() @ w.cpu().double().numpy().T          # exact in 64 bits
    v = sums * (host(sa)[:, None] * host(sw) if scales else 1.0)
    plus = host(b) if bias else 0.0
    if t is torch.float16 and not scales:
        keep = np.abs(v + plus) < 60000
        v, plus, d = np.where(keep, v, 0), np.where(keep, plus, 0), torch.where(torch.from_numpy(keep).cuda(), d, torch.zeros_like(d))
    within("d", d, v + plus, 3.01 * U * np.abs(v) + U * np.abs(v + plus) * (bias is not None), t)
    return d


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 31, 32, 33, 47, 64, 65, 100, 127, 128, 129, 255, 257, 300])
def test_rows(anr, t, M):
    for N, K in ((1, 16), (48, 64), (97, 515), (200, 1363), (129, 17), (33, 31), (16, 2048), (130, 128), (70, 129), (5, 8192)):
        print(t, M, N, K, flush=True)
        case(anr, M, M, N, K, TYPES[t])


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("M", [1, 3, 16, 17, 33, 64, 129, 600])
def test_lengths_of_k(anr, t, M):
    for K in (1, 2, 7, 15, 16, 17, 32, 63, 64, 112, 127, 128, 144, 255, 256, 257, 384, 1000, 1008, 4096, 5000):
        case(anr, 1, M, 77, K, TYPES[t], bias=torch.float32)


@pytest.mark.parametrize("t", TYPES)
def test_tiles(anr, t):
    """Products of many tiles, of few with a long k, and of edges a tile's own and one off."""
    for M, N, K in ((777, 1363, 515), (512, 512, 1024), (513, 511, 640), (1030, 2050, 272), (64, 256, 16384), (200, 300, 20000), (2050, 4100, 144), (4100, 3000, 256), (300, 17000, 130)):
        print(t, M, N, K, flush=True)
        case(anr, 2, M, N, K, TYPES[t], bias=TYPES[t])


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("spare,shift", [(16, 0), (8, 0), (3, 0), (0, 1), (5, 3), (32, 16), (16, 4)])
def test_strides(anr, t, spare, shift):
    for M, N, K in ((1, 50, 160), (20, 100, 200), (40, 64, 128), (300, 270, 400), (7, 9, 11)):
        case(anr, 3, M, N, K, TYPES[t], spare=spare, shift=shift)
        case(anr, 4, M, N, K, TYPES[t], bias=torch.float32, spare=spare, shift=shift, spare_d=8)


@pytest.mark.parametrize("M", [1, 17, 64, 130, 700])
def test_rows_that_start_at_words(anr, M):
    """Leading dimensions of whole words and any k: what lies behind a row's end in its last word, and in the lines behind that, counts for nothing."""
    for N, K, spare in ((70, 515, 1), (70, 513, 3), (33, 1362, 2), (50, 127, 5), (50, 3, 1), (20, 129, 127), (300, 2047, 1), (17, 20001, 3)):
        for shift in (0, 4, 12):
            print(M, N, K, spare, shift, flush=True)
            case(anr, 9, M, N, K, torch.bfloat16, spare=spare, shift=shift + -(spare // 2) % 4, spare_d=0)       # (matrix() starts a row spare // 2 in)


@pytest.mark.parametrize("t", TYPES)
def test_rows_that_start_at_any_byte(anr, t):
    """Odd lengths, each row at another byte of a word, over tiles of every kind, long k that work-groups share, few rows and the longest row offsets in a tile."""
    for M, N, K in ((100, 130, 20001), (200, 300, 16383), (65, 64, 9001), (300, 129, 8195), (2100, 1100, 1030), (1025, 770, 2049), (513, 4100, 259), (40, 9000, 1025), (7, 300, 16385), (1, 4097, 4097)):
        print(t, M, N, K, flush=True)
        case(anr, 10, M, N, K, TYPES[t], bias=TYPES[t], shift=1)
    a, w = (torch.randint(-128, 128, (s, 300001), dtype=torch.int8, device="cuda") for s in (260, 140))
    d = torch.empty(260, 140, dtype=TYPES[t], device="cuda")
    sa, sw = torch.rand(260, device="cuda"), torch.rand(140, device="cuda")
    want = (a[:, 3:1004].cpu().double().numpy() @ w[:, 77777:78778].cpu().double().numpy().T) * (host(sa)[:, None] * host(sw))
    anr.gemm_i8(a[:, 3:1004], w[:, 77777:78778], sa, sw, d)
    if t != "f16":
        within("d", d, want, 3.01 * U * np.abs(want), TYPES[t])


@pytest.mark.parametrize("t", TYPES)
def test_without_scales(anr, t):
    for M, N, K in ((1, 40, 48), (30, 40, 100), (100, 200, 300), (3, 5, 7)):
        case(anr, 5, M, N, K, TYPES[t], scales=False)
        case(anr, 5, M, N, K, TYPES[t], scales=False, bias=TYPES[t])


def test_largest_sums(anr):
    """Products of the largest magnitudes over the longest k: 2^31 - 2^14 in 32 bits."""
    K = (1 << 17) - 1
    for M in (2, 20, 200):
        a, w = torch.full((M, K), -128, dtype=torch.int8, device="cuda"), torch.full((40, K), -128, dtype=torch.int8, device="cuda")
        w[1] = 127
        d = torch.empty(M, 40, device="cuda")
        anr.gemm_i8(a, w, None, None, d)
        assert (d[:, 0] == float(np.float32(128 * 128 * K))).all() and (d[:, 1] == float(np.float32(-128 * 127 * K))).all()
    case(anr, 6, 100, 130, 5000, torch.float32, extreme=True)


def test_exact_sums(anr):
    """Sums below 2^24 come as they are, with scales that are powers of two."""
    r = rng(7)
    for M, N, K in ((1, 300, 600), (17, 300, 600), (90, 300, 600), (400, 700, 1000)):
        a, w = (torch.from_numpy(r.integers(-128, 128, size=s)).to(torch.int8).cuda() for s in ((M, K), (N, K)))
        d = torch.empty(M, N, device="cuda")
        anr.gemm_i8(a, w, torch.full((M,), 0.5, device="cuda"), torch.full((N,), 0.25, device="cuda"), d)
        assert np.array_equal(host(d), a.cpu().double().numpy() @ w.cpu().double().numpy().T / 8)


def test_scales_that_are_not_finite(anr):
    for M in (3, 20, 200):
        a, w, d = torch.ones(M, 64, dtype=torch.int8, device="cuda"), torch.ones(50, 64, dtype=torch.int8, device="cuda"), torch.empty(M, 50, device="cuda")
        sa, sw = torch.ones(M, device="cuda"), torch.ones(50, device="cuda")
        sa[1], sw[7] = float("nan"), float("inf")
        anr.gemm_i8(a, w, sa, sw, d)
        assert torch.isnan(d[1]).all() and (d[0, 7] == float("inf")) and (d[0, :7] == 64).all() and (d[2, 8:] == 64).all()


def test_no_rows(anr):
    e = torch.empty(0, 64, device="cuda")
    anr.gemm_i8(e.char(), torch.ones(8, 64, dtype=torch.int8, device="cuda"), None, None, torch.empty(0, 8, device="cuda"))


def test_one_result_whatever_the_rows(anr):
    """A row's results do not depend on how many rows go with it: the sums are exact."""
    r = rng(8)
    a, w = (torch.from_numpy(r.integers(-128, 128, size=s)).to(torch.int8).cuda() for s in ((700, 1111), (333, 1111)))
    sa, sw = torch.rand(700, device="cuda"), torch.rand(333, device="cuda")
    whole = torch.empty(700, 333, device="cuda")
    anr.gemm_i8(a, w, sa, sw, whole)
    for M in (1, 9, 20, 40, 130, 300):
        d = torch.empty(M, 333, device="cuda")
        anr.gemm_i8(a[:M], w, sa[:M], sw, d)
        assert torch.equal(d, whole[:M])
