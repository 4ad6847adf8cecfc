"""Root-mean-square norm with the residual's addition, its gradients and its form with an output in 8 bits, against their definitions in
64 bits (oracle/blocks.py).

Bounds are those of the arithmetic, with u = 2^-24 and HALF[t] half a step of the type of a result, which is rounded once.  A row's sum of squares is formed by
threads of at most 32 values each, joined over 64 lanes and 16 waves: at most 32 + 6 + 16 roundings one after another and two for h, which rstd
has half of, and four of its own: 32 u.  y takes three more."""
import numpy as np
import pytest

from oracle import blocks as O

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF = {t: torch.finfo(t).eps / 2 for t in TYPES.values()}
TINY = {t: torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2 for t in TYPES.values()}      # half the spacing of denormals
WIDTHS = [1, 2, 3, 5, 7, 8, 9, 63, 64, 65, 100, 255, 512, 515, 768, 1001, 1363, 2048, 4096, 4100, 7001, 16384, 32768]


@pytest.fixture(scope="module")
def anr():
    from paper_2006_06762_amd import binding
    return binding


def rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


def host(t):
    return t.detach().double().cpu().numpy()


def within(name, got, want, bound, t):
    got = host(got)
    assert got.shape == want.shape
    over = np.abs(got - want) - (bound + HALF[t] * (np.abs(want) + bound) + TINY[t])
    at = np.unravel_index(np.argmax(over), over.shape) if over.size else ()
    assert not over.size or np.max(over) <= 0, "%s: %s got %r, want %r, bound %r" % (name, at, got[at], want[at], np.broadcast_to(bound, want.shape)[at])


def matrix(a, t, spare=0, shift=0):
    """[T,C] on the GPU, in the middle of rows that are `spare` longer and begin `shift` elements into their storage; NaN around it."""
    T, C = a.shape
    store = torch.full((T * (C + spare) + shift,), float("nan") if t.is_floating_point else 77, dtype=t, device="cuda")
    view = store[shift:].view(T, C + spare)[:, spare // 2:spare // 2 + C]
    view.copy_(torch.from_numpy(np.ascontiguousarray(a)))
    return view


def untouched(view):
    """Whether what lies around a matrix() is as it was."""
    store = torch.as_strided(view, (view.untyped_storage().nbytes() // view.element_size(),), (1,), 0).clone()
    seen = torch.zeros(store.shape, dtype=torch.bool, device="cuda")
    torch.as_strided(seen, view.shape, view.stride(), view.storage_offset()).fill_(True)
    rest = store[~seen]
    return bool(torch.isnan(rest).all() if rest.is_floating_point() else (rest == 77).all())


def make(seed, T, C, t, param, spare=0, shift=0):
    r = rng(seed)
    size = np.where(r.uniform(size=C) < 0.02, 8.0, 1.0) * r.uniform(0.5, 1.5, size=(T, 1))
    gamma = torch.from_numpy(r.normal(size=C) * 0.3 + 1).to(param).cuda()
    return r, matrix(r.normal(size=(T, C)) * size, t, spare, shift), matrix(r.normal(size=(T, C)), t, spare, shift), gamma


def forward_case(anr, seed, T, C, t, residual, param=None, spare=0, shift=0, eps=1e-6):
    param = param or t
    r, x, res, gamma = make(seed, T, C, t, param, spare, shift)
    blank = np.full((T, C), np.nan)
    y, h = matrix(blank, t, spare, shift), matrix(blank, t, spare, shift) if residual else None
    rstd = torch.full((T,), float("nan"), device="cuda")
    before = x.clone(), res.clone()
    assert anr.rms_norm(x, y, gamma, eps, res if residual else None, h, rstd) is y
    wh, wy, wr = O.rms_norm(host(x), host(res) if residual else None, host(gamma), eps)
    within("rstd", rstd, wr, 32 * U * wr, torch.float32)
    within("y", y, wy, 35 * U * np.abs(wy), t)
    if residual:
        within("h", h, wh, U * np.abs(wh), t)
    assert torch.equal(x, before[0]) and torch.equal(res, before[1]) and all(untouched(v) for v in (x, res, y))

    q, scale = matrix(np.zeros((T, C)), torch.int8, spare, shift), torch.full((T,), float("nan"), device="cuda")
    h2 = matrix(blank, t, spare, shift) if residual else None
    got = anr.rms_norm_q8(x, q, scale, gamma, eps, res if residual else None, h2)
    assert got[0] is q and got[1] is scale and untouched(q) and (not residual or torch.equal(h2, h))
    steps, ws = O.in_8_bits(wy)
    within("scale", scale, ws, 36 * U * ws, torch.float32)
    # q of h gamma (rounded twice) times the inverse of the step (twice more, the product once)
    assert np.all(np.abs(host(q) - steps) <= 0.5 + 127 * 6 * U)
    assert np.all(np.abs(host(q)).max(1) == 127)
    return x, y, h


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("C", WIDTHS)
def test_forward_widths(anr, t, C):
    for T in (1, 3, 6) if C > 4096 else (1, 2, 37, 1030):
        print(t, T, C, flush=True)
        forward_case(anr, 1, T, C, TYPES[t], True)
    forward_case(anr, 2, 5, C, TYPES[t], False, torch.float32)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("spare,shift", [(8, 0), (3, 0), (0, 1), (5, 3), (16, 8)])
def test_forward_strides(anr, t, spare, shift):
    for T, C in ((9, 40), (1025, 264), (2, 1363), (3, 6)):
        forward_case(anr, 3, T, C, TYPES[t], True, spare=spare, shift=shift)


def backward_case(anr, seed, T, C, t, extra, param=None, spare=0, shift=0):
    param = param or t
    r, x, dh, gamma = make(seed, T, C, t, param, spare, shift)
    dy = matrix(r.normal(size=(T, C)), t, spare, shift)
    rstd = torch.from_numpy(O.rms_norm(host(x), None, 1.0, 1e-6)[2]).float().cuda()
    dx, dgamma = matrix(np.full((T, C), np.nan), t, spare, shift), torch.full((C,), float("nan"), dtype=param, device="cuda")
    got = anr.rms_norm_backward(dy, x, gamma, rstd, dx, dgamma, dh if extra else None)
    assert got[0] is dx and got[1] is dgamma and untouched(dx)
    wx, wg, hat, size = O.rms_norm_backward(host(dy), host(x), host(gamma), host(rstd), host(dh) if extra else None)
    g, s = np.abs(host(dy) * host(gamma)), host(rstd)[:, None]
    # the mean of n products of three roundings each, as rstd's; then a product, a difference and two products, and the sum with dh
    within("dx", dx, wx, s * (6 * U * g + np.abs(hat) * (62 + 6) * U * size) + 2 * U * np.abs(wx), t)
    # rows one after another in a work-group, then its rows, then the work-groups in 32 runs
    within("dgamma", dgamma, wg, (T / 512 + 4 + 16 + 32 + 4) * U * np.abs(host(dy) * hat).sum(0), param)
    alone = torch.full_like(dgamma, float("nan"))
    anr.rms_norm_backward(dy, x, gamma, rstd, None, alone)
    assert torch.equal(alone, dgamma)
    again = matrix(np.full((T, C), np.nan), t, spare, shift)
    anr.rms_norm_backward(dy, x, gamma, rstd, again, None, dh if extra else None)
    assert torch.equal(again, dx)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("C", WIDTHS)
def test_backward_widths(anr, t, C):
    for T in (1, 3, 6) if C > 4096 else (1, 2, 37, 1030):
        print(t, T, C, flush=True)
        backward_case(anr, 4, T, C, TYPES[t], True)
    backward_case(anr, 5, 5, C, TYPES[t], False, torch.float32)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("spare,shift", [(8, 0), (3, 0), (0, 1), (5, 3)])
def test_backward_strides(anr, t, spare, shift):
    for T, C in ((9, 40), (1025, 264), (2, 1363), (3, 6)):
        backward_case(anr, 6, T, C, TYPES[t], True, spare=spare, shift=shift)


@pytest.mark.parametrize("t", TYPES)
def test_many_rows(anr, t):
    """More rows than a backward pass has work-groups."""
    forward_case(anr, 7, 5003, 136, TYPES[t], True, torch.float32)
    backward_case(anr, 7, 5003, 136, TYPES[t], True, torch.float32)
    backward_case(anr, 7, 2100, 1100, TYPES[t], False, torch.float32)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("C", [5, 264, 1363, 4096])
def test_in_place(anr, t, C):
    T, t = 19, TYPES[t]
    _, x, res, gamma = make(8, T, C, t, t)
    y, h = torch.empty_like(x), torch.empty_like(x)
    anr.rms_norm(x, y, gamma, 1e-6, res, h)
    for hx in (True, False):                     # the sum over x or over the residual, the result over the other one
        a, b = x.clone(), res.clone()
        anr.rms_norm(a, b if hx else a, gamma, 1e-6, b, a if hx else b)
        assert torch.equal(a if hx else b, h) and torch.equal(b if hx else a, y)
    a, b = x.clone(), res.clone()
    q, scale, q2, scale2 = (torch.empty(s, dtype=d, device="cuda") for _ in range(2) for s, d in (((T, C), torch.int8), ((T,), torch.float32)))
    anr.rms_norm_q8(x, q, scale, gamma, 1e-6, res)
    anr.rms_norm_q8(a, q2, scale2, gamma, 1e-6, b, b)
    assert torch.equal(b, h) and torch.equal(q, q2) and torch.equal(scale, scale2)
    dy, rstd = torch.randn(T, C, device="cuda").to(t), torch.rand(T, device="cuda") + 0.5
    dx, dgamma = torch.empty_like(x), torch.empty_like(gamma)
    anr.rms_norm_backward(dy, x, gamma, rstd, dx, dgamma, res)
    for which in range(3):
        ins, dg = [dy.clone(), x.clone(), res.clone()], torch.empty_like(gamma)
        anr.rms_norm_backward(ins[0], ins[1], gamma, rstd, ins[which], dg, ins[2])
        assert torch.equal(ins[which], dx) and torch.equal(dg, dgamma)


def test_absent_gamma_is_ones(anr):
    for t in TYPES.values():
        _, x, res, _ = make(9, 33, 515, t, t)
        ones = torch.ones(515, dtype=t, device="cuda")
        outs = []
        for g in (None, ones):
            y, q, scale, dx, dg = torch.empty_like(x), torch.empty(33, 515, dtype=torch.int8, device="cuda"), torch.empty(33, device="cuda"), torch.empty_like(x), torch.empty_like(ones)
            anr.rms_norm(x, y, g, 1e-6, res)
            anr.rms_norm_q8(x, q, scale, g, 1e-6, res)
            anr.rms_norm_backward(res, x, g, scale, dx, dg)
            outs.append((y, q, scale, dx, dg))
        assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_no_rows(anr):
    x = torch.empty(0, 64, device="cuda")
    none = torch.empty(0, device="cuda")
    anr.rms_norm(x, x.clone(), rstd=none)
    anr.rms_norm_q8(x, x.char(), none)
    dg = torch.full((64,), float("nan"), device="cuda")
    anr.rms_norm_backward(x, x, None, none, x.clone(), dg)
    assert torch.equal(dg, torch.zeros_like(dg))


def test_special_values(anr):
    C = 300
    x = torch.randn(8, C, device="cuda")
    x[1] = 0
    x[2, 7] = float("nan")
    x[3, 299] = float("inf")
    x[4] *= 1e-38                               # squares below float32's range: eps alone
    x[5] *= 1e15
    x[6, 5] = -float("inf")
    y, q, scale, rstd = torch.empty_like(x), torch.empty(8, C, dtype=torch.int8, device="cuda"), torch.empty(8, device="cuda"), torch.empty(8, device="cuda")
    anr.rms_norm(x, y, None, 1e-6, rstd=rstd)
    anr.rms_norm_q8(x, q, scale, None, 1e-6)
    for row in (0, 4, 5, 7):
        want = O.rms_norm(host(x[row:row + 1]), None, 1.0, 1e-6)
        within("y", y[row:row + 1], want[1], 35 * U * np.abs(want[1]), torch.float32)
        steps, ws = O.in_8_bits(want[1])
        within("scale", scale[row:row + 1], ws, 36 * U * ws, torch.float32)
        assert np.all(np.abs(host(q[row:row + 1]) - steps) <= 0.5 + 127 * 6 * U)
    assert (y[1] == 0).all() and (q[1] == 0).all() and scale[1] == 0
    assert torch.isnan(y[2]).all()
    for row in (2, 3, 6):
        assert (q[row] == 0).all() and torch.isnan(scale[row])


def test_gradients_against_differences(anr):
    """The gradient of sum(y w) + sum(h v), by central differences of the definition in 64 bits."""
    T, C, eps = 3, 20, 1e-3
    r = rng(10)
    x, res, gamma, w, v = (r.normal(size=s).astype(np.float32).astype(np.float64) for s in ((T, C), (T, C), (C,), (T, C), (T, C)))
    f = lambda a, b, g: (O.rms_norm(a, b, g, eps)[1] * w).sum() + ((a + b) * v).sum()  # noqa: E731
    dev = lambda a: torch.from_numpy(a).float().cuda()  # noqa: E731
    h, y, rstd, dx, dg = torch.empty(T, C, device="cuda"), torch.empty(T, C, device="cuda"), torch.empty(T, device="cuda"), torch.empty(T, C, device="cuda"), torch.empty(C, device="cuda")
    anr.rms_norm(dev(x), y, dev(gamma), eps, dev(res), h, rstd)
    anr.rms_norm_backward(dev(w), h, dev(gamma), rstd, dx, dg, dev(v))
    step = 1e-4
    for i in range(T):
        for c in range(0, C, 3):
            e = np.zeros((T, C))
            e[i, c] = step
            slope = (f(x + e, res, gamma) - f(x - e, res, gamma)) / (2 * step)
            assert abs(slope - (f(x, res + e, gamma) - f(x, res - e, gamma)) / (2 * step)) < 1e-7
            assert abs(float(dx[i, c]) - slope) < 1e-5 * (1 + abs(slope))
    for c in range(C):
        e = np.zeros(C)
        e[c] = step
        slope = (f(x, res, gamma + e) - f(x, res, gamma - e)) / (2 * step)
        assert abs(float(dg[c]) - slope) < 1e-5 * (1 + abs(slope))


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_largest_magnitudes(anr, t):
    """Rows of 2^56 all over, whose squares sum to 2^127 at the most: powers of two, exact throughout."""
    t = TYPES[t]
    for C in (300, 32768):
        sign = torch.from_numpy(rng(11).choice([-1.0, 1.0], size=(3, C)))
        for share in (1.0, 0.5):                 # of the sum that x has
            x, res = (sign * 2.0 ** 56 * share).to(t).cuda(), (sign * 2.0 ** 56 * (1 - share)).to(t).cuda()
            y, h, q, scale = torch.empty_like(x), torch.empty_like(x), torch.empty(3, C, dtype=torch.int8, device="cuda"), torch.empty(3, device="cuda")
            anr.rms_norm(x, y, None, 0.0, res, h)
            anr.rms_norm_q8(x, q, scale, None, 0.0, res)
            # (every partial sum is at most 2^15 times a power of two, the mean is 2^112, its root and that one's inverse are powers of two)
            assert np.array_equal(host(y), sign.numpy()) and np.array_equal(host(h), sign.numpy() * 2.0 ** 56)
            assert np.array_equal(host(q), 127 * sign.numpy()) and (scale == np.float32(1) / np.float32(127)).all()


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("C", [9001, 16385, 20001, 32767])
def test_wide_ragged_rows(anr, t, C):
    """Rows of more units than a work-group has threads, whose last unit begins inside another one's; more of them than work-groups; in place."""
    t = TYPES[t]
    forward_case(anr, 12, 3, C, t, True)
    for T in (2, 300):
        print(t, T, C, flush=True)
        backward_case(anr, 12, T, C, t, True)
        backward_case(anr, 13, T, C, t, False, torch.float32, spare=3, shift=1)
    _, x, dh, gamma = make(14, 5, C, t, t)
    dy, rstd = torch.randn(5, C, device="cuda").to(t), torch.rand(5, device="cuda") + 0.5
    dx, dgamma = torch.empty_like(x), torch.empty_like(gamma)
    anr.rms_norm_backward(dy, x, gamma, rstd, dx, dgamma, dh)
    for which in range(3):
        ins, dg = [dy.clone(), x.clone(), dh.clone()], torch.empty_like(gamma)
        anr.rms_norm_backward(ins[0], ins[1], gamma, rstd, ins[which], dg, ins[2])
        assert torch.equal(ins[which], dx) and torch.equal(dg, dgamma)
