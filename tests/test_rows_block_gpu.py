"""The operators together, as a block runs them: a feed-forward block in 8 bits behind a residual, with gate's and up's weights as one matrix, for prompts and
single tokens, captured too; a training step through norm and feed-forward block against the gradients of the formulas in 64 bits; operands and results whose
offsets pass 32 bits."""
import numpy as np
import pytest

from oracle import blocks as O
from tests.test_rms_norm_gpu import HALF, U, host, rng

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def anr():
    from paper_2006_06762_amd import binding
    return binding


def dev(a, t=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(t).cuda()


class Block:
    """h = x + residual; y = (act(norm(h) w_gate^T) * (norm(h) w_up^T)) w_down^T with weights and tokens in 8 bits."""

    def __init__(self, anr, C, F, t, seed):
        r = rng(seed)
        self.anr, self.t, self.C, self.F = anr, t, C, F
        self.gamma = dev(r.normal(size=C) * 0.2 + 1, t)
        both, down = dev(r.normal(size=(2 * F, C)) / np.sqrt(C)), dev(r.normal(size=(C, F)) / np.sqrt(F))
        e = lambda *s, d=torch.float32: torch.empty(s, dtype=d, device="cuda")  # noqa: E731
        self.w = e(2 * F, C, d=torch.int8), e(2 * F)
        self.down = e(C, F, d=torch.int8), e(C)
        anr.quantize_rows(both, *self.w)
        anr.quantize_rows(down, *self.down)
        self.exact = host(both), host(down)

    def buffers(self, T):
        e = lambda *s, d=self.t: torch.empty(s, dtype=d, device="cuda")  # noqa: E731
        C, F = self.C, self.F
        return {"h": e(T, C), "q": e(T, C, d=torch.int8), "s": e(T, d=torch.float32), "gu": e(T, 2 * F), "q2": e(T, F, d=torch.int8), "s2": e(T, d=torch.float32), "y": e(T, C)}

    def __call__(self, x, residual, b):
        anr, F = self.anr, self.F
        anr.rms_norm_q8(x, b["q"], b["s"], self.gamma, 1e-6, residual, b["h"])
        anr.gemm_i8(b["q"], self.w[0], b["s"], self.w[1], b["gu"])
        anr.quantize_rows(b["gu"][:, :F], b["q2"], b["s2"], anr.ANR_ACT_SILU, b["gu"][:, F:])
        anr.gemm_i8(b["q2"], self.down[0], b["s2"], self.down[1], b["y"])
        return b


@pytest.mark.parametrize("t", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("T,C,F", [(1, 256, 688), (30, 96, 200), (50, 515, 1363), (300, 512, 1408)])
def test_feed_forward_in_8_bits(anr, t, T, C, F):
    """Each stage against the definition of it from what the stage before left, and the whole against the block on exact weights: a value in 8 bits is off by half a step at most, a
    product by what its operands are off."""
    block = Block(anr, C, F, t, 1)
    r = rng(2)
    x, res = dev(r.normal(size=(T, C)), t), dev(r.normal(size=(T, C)), t)
    b = {k: host(v) for k, v in block(x, res, block.buffers(T)).items()}
    _, y, _ = O.rms_norm(host(x), host(res), host(block.gamma), 1e-6)
    back = b["q"] * b["s"][:, None]
    assert np.all(np.abs(back - y) <= (0.5 + 127 * 50 * U) * b["s"][:, None])
    w = host(block.w[0]) * host(block.w[1])[:, None]
    gu = back @ w.T
    half = HALF[t]
    assert np.all(np.abs(b["gu"] - gu) <= (4 * U + half) * np.abs(gu) * (1 + 4 * U) + 1e-7)
    g, u = b["gu"][:, :F], b["gu"][:, F:]
    v = O.act("silu", g)[0] * u
    back2 = b["q2"] * b["s2"][:, None]
    # (silu to 64 u of 1 + |g|)
    assert np.all(np.abs(back2 - v) <= (0.5 + 127 * 8 * U) * b["s2"][:, None] + 66 * U * (1 + np.abs(g)) * np.abs(u) * 2)
    wd = host(block.down[0]) * host(block.down[1])[:, None]
    out = back2 @ wd.T
    assert np.all(np.abs(b["y"] - out) <= (4 * U + half) * np.abs(out) * (1 + 4 * U) + 1e-7)
    # the whole: errors of values (half a step), of weights (half a step of theirs), through |silu'| <= 1.1
    wide = 1.01
    ey = 0.51 * b["s"][:, None] * np.ones_like(y)
    ew, ed = 0.51 * host(block.w[1])[:, None], 0.51 * host(block.down[1])[:, None]
    e_gu = (ey @ np.abs(w).T + np.abs(y) @ (ew * np.ones_like(w)).T) * wide + half * np.abs(gu)
    want_g, want_u = y @ block.exact[0][:F].T, y @ block.exact[0][F:].T
    eg, eu = e_gu[:, :F], e_gu[:, F:]
    assert np.all(np.abs(g - want_g) <= eg + 1e-5) and np.all(np.abs(u - want_u) <= eu + 1e-5)
    want_v = O.act("silu", want_g)[0] * want_u
    ev = 1.1 * eg * (np.abs(want_u) + eu) + np.abs(O.act("silu", want_g)[0]) * eu + 0.51 * b["s2"][:, None]
    want = want_v @ block.exact[1].T
    e_out = (ev @ np.abs(wd).T + np.abs(want_v) @ (ed * np.ones_like(wd)).T) * wide + half * np.abs(out)
    assert np.all(np.abs(b["y"] - want) <= e_out + 1e-5)
    # (and nearer than the worst case by far: errors of opposite signs cancel)
    assert np.linalg.norm(b["y"] - want) <= 0.05 * np.linalg.norm(want)


def test_captured_single_tokens(anr):
    """One token a step with the sum going on in place, in a graph, against the same steps made eagerly."""
    t, C, F = torch.bfloat16, 256, 688
    block = Block(anr, C, F, t, 3)
    start, steps = dev(rng(4).normal(size=(1, C)), t), 5
    b = block.buffers(1)
    x, res = torch.zeros(1, C, dtype=t, device="cuda"), start.clone()

    def step():
        anr.rms_norm_q8(x, b["q"], b["s"], block.gamma, 1e-6, res, res)         # the residual stream in place
        anr.gemm_i8(b["q"], block.w[0], b["s"], block.w[1], b["gu"])
        anr.quantize_rows(b["gu"][:, :F], b["q2"], b["s2"], anr.ANR_ACT_SILU, b["gu"][:, F:])
        anr.gemm_i8(b["q2"], block.down[0], b["s2"], block.down[1], x)
    want = []
    for _ in range(steps):
        step()
        want.append((x.clone(), res.clone()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        x.zero_(), res.copy_(start)
        for wx, wr in want:
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(x, wx) and torch.equal(res, wr)
            torch.randn(1000, device="cuda").sum().item()


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
def test_training_step(anr, t):
    """out = h + ff(norm(h)), h = x + residual: gradients of sum(out w) for x, gamma and the weights, against automatic differentiation in 64 bits."""
    T, C, F = 70, 96, 176
    r = rng(5)
    x, res, w = (dev(r.normal(size=(T, C)), t) for _ in range(3))
    gamma = dev(r.normal(size=C) * 0.2 + 1, torch.float32)
    wg, wu, wd = dev(r.normal(size=(F, C)) / 10, t), dev(r.normal(size=(F, C)) / 10, t), dev(r.normal(size=(C, F)) / 13, t)
    e = torch.empty_like
    h, y, rstd, z = e(x), e(x), torch.empty(T, device="cuda"), e(x)
    gate, up = (torch.empty(T, F, dtype=t, device="cuda") for _ in range(2))
    anr.rms_norm(x, y, gamma, 1e-6, res, h, rstd)
    anr.gated_ff(y, wg, wu, wd, z, anr.ANR_ACT_SILU, gate, up)
    dy, dx, dgamma, dwg, dwu, dwd = e(x), e(x), e(gamma), e(wg), e(wu), e(wd)
    anr.gated_ff_backward(w, y, wg, wu, wd, gate, up, dy, dwg, dwu, dwd, anr.ANR_ACT_SILU)
    anr.rms_norm_backward(dy, h, gamma, rstd, dx, dgamma, w)
    leaves = [v.double().cpu().requires_grad_() for v in (x, gamma, wg, wu, wd)]
    lx, lg, lwg, lwu, lwd = leaves
    hh = lx + res.double().cpu()
    yy = hh * torch.rsqrt(hh.square().mean(1, keepdim=True) + 1e-6) * lg
    g = yy @ lwg.t()
    out = hh + (g * torch.sigmoid(g) * (yy @ lwu.t())) @ lwd.t()
    want = torch.autograd.grad((out * w.double().cpu()).sum(), leaves)
    # six roundings to the type between x and a gradient (h, y, gate and up, the hidden gradients, dy, the result), each of which moves it by at most its own size
    # relative to the gradient's norm; in float32 sums of up to 176 products of random signs come on top, 16 roundings of them
    bound = 6 * HALF[t] + 16 * U
    for name, got, ref in zip(("x", "gamma", "w_gate", "w_up", "w_down"), (dx, dgamma, dwg, dwu, dwd), want):
        off = float((got.double().cpu() - ref).norm() / ref.norm())
        assert off <= bound, (name, off, bound)


def test_offsets_beyond_32_bits(anr):
    """Rows far apart: operands and results of more than 4 GiB between the first and the last."""
    r = rng(6)
    far = (1 << 22) - 64
    for M in (9, 40, 1100):
        store = torch.empty(M * far, dtype=torch.int8, device="cuda")
        a = store.view(M, far)[:, :192]
        a.copy_(dev(r.integers(-128, 128, size=(M, 192)), torch.int8))
        w = dev(r.integers(-128, 128, size=(70, 192)), torch.int8)
        d = torch.empty(M, 70, device="cuda")
        anr.gemm_i8(a, w, None, None, d)
        want = host(a) @ host(w).T
        assert np.array_equal(host(d), want)
        anr.gemm_i8(w, a, None, None, d.view(-1).view(70, M))
        assert np.array_equal(host(d.view(-1).view(70, M)), want.T)
        del store, a
    T, C, ld = 1200, 40, 1 << 21
    store = torch.empty(T * ld, dtype=torch.bfloat16, device="cuda")
    x, y = store.view(T, ld)[:, :C], store.view(T, ld)[:, 1000:1000 + C]
    x.copy_(dev(r.normal(size=(T, C)), torch.bfloat16))
    packed, g, rstd = x.clone(), dev(r.normal(size=C)), torch.empty(T, device="cuda")
    want, rw = torch.empty_like(packed), torch.empty_like(rstd)
    anr.rms_norm(x, y, g, 1e-6, rstd=rstd)
    anr.rms_norm(packed, want, g, 1e-6, rstd=rw)
    assert torch.equal(y, want) and torch.equal(rstd, rw)
    dg, dgw, dw = torch.empty_like(g), torch.empty_like(g), torch.empty_like(packed)
    anr.rms_norm_backward(packed, packed, g, rstd, dw, dgw)
    anr.rms_norm_backward(x, x, g, rstd, y, dg)
    assert torch.equal(y, dw) and torch.equal(dg, dgw)
    q, s, qw, sw = torch.empty(T, C, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda"), torch.empty(T, C, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    anr.quantize_rows(x, q, s)
    anr.quantize_rows(packed, qw, sw)
    assert torch.equal(q, qw) and torch.equal(s, sw)
    anr.dequantize_rows(q, s, y)
    anr.dequantize_rows(qw, sw, dw)
    assert torch.equal(y, dw)


def test_more_rows_than_a_launch_has_work_groups(anr):
    """Millions of short rows: what a launch's work-groups take in turn."""
    T, C = (1 << 22) + 77, 3
    x = torch.randn(T, C, device="cuda")
    y, q, s, back = torch.empty_like(x), torch.empty(T, C, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda"), torch.empty_like(x)
    anr.rms_norm(x, y)
    want = x.double() * torch.rsqrt(x.double().square().mean(1, keepdim=True) + 1e-6)
    assert float(((y.double() - want).abs() / (want.abs() + 1e-30)).max()) <= 36 * U
    anr.quantize_rows(x, q, s)
    anr.dequantize_rows(q, s, back)
    assert bool(((back.double() - x.double()).abs() <= (0.5 + 127 * 8 * U) * s.double()[:, None]).all())
    dx, dg = torch.empty_like(x), torch.empty(C, device="cuda")
    ones = torch.ones(T, device="cuda")
    anr.rms_norm_backward(x, x, None, ones, dx, dg)
    sums = x.double().square().sum(0)
    # (rows one after another in a thread, 2^22 over 2^15 of them, then the work-groups' joins)
    assert float(((dg.double() - sums).abs() / sums).max()) <= (T / 2 ** 15 + 200) * U


def test_rows_behind_the_last_stay(anr):
    """A batch that fills part of its buffers."""
    T, C, N = 21, 136, 50
    x, y = torch.randn(40, C, device="cuda"), torch.full((40, C), 7.0, device="cuda")
    q, s, d = torch.full((40, C), 7, dtype=torch.int8, device="cuda"), torch.full((40,), 7.0, device="cuda"), torch.full((40, N), 7.0, device="cuda")
    w = torch.ones(N, C, dtype=torch.int8, device="cuda")
    anr.rms_norm(x[:T], y[:T])
    anr.rms_norm_q8(x[:T], q[:T], s[:T])
    anr.gemm_i8(q[:T], w, s[:T], None, d[:T])
    for v in (y, q, s, d):
        assert (v[T:] == 7).all() and not (v[:T] == 7).all()
