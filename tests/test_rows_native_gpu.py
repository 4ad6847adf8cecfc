"""The extension module's root-mean-square norm, rows in 8 bits and their products against the Python functions it stands before: the same results for every way to
pass the arguments, and the same errors; calls of threads, on streams and in captures."""
import threading

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

NAMES = ["rms_norm", "rms_norm_q8", "rms_norm_backward", "quantize_rows", "dequantize_rows", "gemm_i8"]


@pytest.fixture(scope="module")
def anr():
    from paper_2006_06762_amd import binding
    return binding


def rand(*shape, t=torch.float32):
    return (torch.rand(shape, device="cuda") - 0.5).to(t)


def whole(*shape):
    return torch.randint(-128, 128, shape, device="cuda").to(torch.int8)


def calls(anr, name):
    """(args, kwargs, outputs) of calls that the extension module takes and of some that go to Python."""
    out = []
    for t in (torch.float32, torch.float16, torch.bfloat16):
        T, C = 19, 136
        x, r, h, y, dy, dx, dh = (rand(T, C, t=t) for _ in range(7))
        wide = [rand(T, C + 5, t=t)[:, 2:C + 2] for _ in range(2)]
        g, dg, gf, dgf = rand(C, t=t), rand(C, t=t), rand(C), rand(C)
        s, q, qw = rand(T).abs() + 0.5, whole(T, C), whole(T, C + 3)[:, :C]
        if name == "rms_norm":
            out += [((x, y), {}, [y]), ((x, y, g, 1e-3), {"residual": r, "h": h, "rstd": s}, [y, h, s]), ((x, y, gf, 1e-5, r, None, None), {}, [y]),
                    ((wide[0],), {"y": wide[1], "gamma": gf}, [wide[1]]), ((x, y, None, 1), {}, [y]), ((x[:1], y[:1], g), {}, [y[:1]])]
        elif name == "rms_norm_q8":
            out += [((x, q, s), {}, [q, s]), ((x, qw, s, gf, 1e-5, r, h), {}, [qw, s, h]), ((wide[0], q), {"scale": s, "gamma": g, "residual": wide[1]}, [q, s]), ((x, q, s, None, 0), {}, [q, s])]
        elif name == "rms_norm_backward":
            out += [((dy, x, g, s, dx, dg, dh), {}, [dx, dg]), ((dy, x, gf, s), {"dx": dx, "dgamma": dgf}, [dx, dgf]), ((dy, x, None, s, None, dg), {}, [dg]), ((wide[0], x, g, s, wide[1]), {}, [wide[1]]),
                    ((dy, x, g, s, dx, dg), {"ws": torch.empty(1 << 20, dtype=torch.uint8, device="cuda")}, [dx, dg]), ((dy, x, None, s), {"dgamma": dgf, "dh": dh, "dx": dx}, [dx, dgf])]
        elif name == "quantize_rows":
            out += [((x, q, s), {}, [q, s]), ((x, q, s, anr.ANR_ACT_SILU, r), {}, [q, s]), ((wide[0], qw, s), {"up": wide[1], "act": 3}, [qw, s]), ((x, q, s, True), {}, [q, s])]
        elif name == "dequantize_rows":
            out += [((q, s, y), {}, [y]), ((qw,), {"scale": s, "y": wide[0]}, [wide[0]]), ((q[:1], s[:1], y[:1]), {}, [y[:1]])]
        else:
            for M in (1, 19, 300):
                a, w, wl = whole(M, 272), whole(96, 272), whole(96, 275)[:, 1:273]
                sa, sw, b, bf, d, dl = rand(M), rand(96), rand(96, t=t), rand(96), rand(M, 96, t=t), rand(M, 99, t=t)[:, :96]
                out += [((a, w, sa, sw, d), {}, [d]), ((a, wl, None, sw), {"d": dl, "bias": b}, [dl]), ((a, w, sa, None, d, bf, None), {}, [d]),
                        ((a, w, sa, sw, d), {"bias": bf, "ws": torch.empty(1 << 22, dtype=torch.uint8, device="cuda")}, [d])]
            a, w, sa, sw, d = whole(200, 20000), whole(64, 20000), rand(200), rand(64), rand(200, 64, t=t)
            out += [((a, w, sa, sw, d), {}, [d])]
    return out


def blank(o):
    o.fill_(float("nan") if o.is_floating_point() else 77)


@pytest.mark.parametrize("name", NAMES)
def test_same_results(anr, name):
    for args, kwargs, outs in calls(anr, name):
        for o in outs:
            blank(o)
        python = getattr(anr, "_" + name)(*args, **kwargs)
        want = [o.clone() for o in outs]
        assert not any(torch.isnan(w).any() for w in want if w.is_floating_point())
        for on in (torch.cuda.current_stream(), torch.cuda.Stream()):
            for o in outs:
                blank(o)
            on.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(on):
                native = getattr(anr, name)(*args, **kwargs)
            torch.cuda.synchronize()
            assert all(torch.equal(o, w) for o, w in zip(outs, want))
            assert type(native) is type(python)
            assert native is python if not isinstance(python, tuple) else all(a is b for a, b in zip(native, python)) and len(native) == len(python)


def test_same_errors(anr):
    x, y, h, s, g, q = rand(6, 8), rand(6, 8), rand(6, 8), rand(6), rand(8), whole(6, 8)
    w, sw, d = whole(5, 8), rand(5), rand(6, 5)
    flat, line = rand(48), rand(1, 8).expand(6, 8)
    bad = [("rms_norm", (x,), {}), ("rms_norm", (x, y[:5]), {}), ("rms_norm", (x, y.half()), {}), ("rms_norm", (x, y, s), {}), ("rms_norm", (x, y, g.half()), {}), ("rms_norm", (x, y, g, -1.0), {}),
           ("rms_norm", (x, y, g, "eps"), {}), ("rms_norm", (x, y), {"h": h}), ("rms_norm", (x, y), {"residual": h, "h": y}), ("rms_norm", (x, y), {"rstd": g}), ("rms_norm", (x, y.cpu()), {}),
           ("rms_norm", (flat, flat), {}), ("rms_norm", (x, line), {}), ("rms_norm", (line, y), {}), ("rms_norm", (x.t(), y.t()), {}), ("rms_norm", (x, y), {"gama": g}), ("rms_norm", (q, y), {}), ("rms_norm", (x, None), {}),
           ("rms_norm_q8", (x, q), {}), ("rms_norm_q8", (x, y, s), {}), ("rms_norm_q8", (x, q, s.half()), {}), ("rms_norm_q8", (x, q, g), {}), ("rms_norm_q8", (x, q, None), {}), ("rms_norm_q8", (x, q, s), {"h": h}),
           ("rms_norm_q8", (x, q, s, g, float("nan")), {}), ("rms_norm_backward", (x, y, g, s), {}), ("rms_norm_backward", (x, y, g, None, h), {}), ("rms_norm_backward", (x, y, g, g, h), {}),
           ("rms_norm_backward", (x, y, g, s, h, g.half()), {}), ("rms_norm_backward", (None, y, g, s, h), {}), ("rms_norm_backward", (x, y, g, s, h[:3]), {}),
           ("rms_norm_backward", (x, y, g, s, h, g), {"ws": torch.empty(4, dtype=torch.uint8, device="cuda")}),
           ("quantize_rows", (x, q), {}), ("quantize_rows", (x, y, s), {}), ("quantize_rows", (x, q, g), {}), ("quantize_rows", (x, q, s, 9), {}), ("quantize_rows", (x, q, s, 0, y[:2]), {}), ("quantize_rows", (q, q, s), {}),
           ("quantize_rows", (line, q, None), {}), ("dequantize_rows", (q, s), {}), ("dequantize_rows", (y, s, x), {}), ("dequantize_rows", (q, g, x), {}), ("dequantize_rows", (q, s, q), {}), ("dequantize_rows", (q, None, x), {}),
           ("gemm_i8", (q, w, s, sw), {}), ("gemm_i8", (q, w[:, :7], s, sw, d), {}), ("gemm_i8", (q, w, sw, s, d), {}), ("gemm_i8", (q, w, s, sw, d.t()), {}), ("gemm_i8", (x, w, s, sw, d), {}),
           ("gemm_i8", (q, w, s, sw, d, sw.half()), {}), ("gemm_i8", (q, w, s, sw, d, s), {}), ("gemm_i8", (q, w, s, sw, d.double()), {}), ("gemm_i8", (q, w, s, sw, d, 3), {}), ("gemm_i8", (q, w.cpu(), s, sw, d), {}),
           ("gemm_i8", (q, w, s.double(), sw, d), {}), ("gemm_i8", (whole(200, 20000), whole(64, 20000), None, None, rand(200, 64)), {"ws": torch.empty(64, dtype=torch.uint8, device="cuda")})]
    for name, args, kwargs in bad:
        raised = []
        for prefix in ("", "_"):
            with pytest.raises(Exception) as e:
                getattr(anr, prefix + name)(*args, **kwargs)
            raised.append((type(e.value), str(e.value)))
        assert raised[0] == raised[1], (name, args, kwargs, raised)


def test_parameters_and_subclasses(anr):
    """Weights as torch.nn.Parameter, and a tensor subclass, which goes to Python."""
    class Sub(torch.Tensor):
        pass

    x, y, g = rand(20, 16), rand(20, 16), rand(16)
    want = anr._rms_norm(x, y, g).clone()
    assert torch.equal(anr.rms_norm(x, y.zero_(), torch.nn.Parameter(g)), want)
    assert torch.equal(anr.rms_norm(x.as_subclass(Sub), y.zero_(), g), want)


def jobs(anr):
    """Calls of two launches on workspaces: (run, outputs)."""
    dy, x, g, s = rand(3000, 512, t=torch.bfloat16), rand(3000, 512, t=torch.bfloat16), rand(512), rand(3000).abs()
    dx, dg = torch.empty_like(x), torch.empty_like(g)
    a, w, sa, sw, d = whole(150, 12000), whole(128, 12000), rand(150), rand(128), torch.empty(150, 128, device="cuda")

    def run(dx=dx, dg=dg, d=d):
        anr.rms_norm_backward(dy, x, g, s, dx, dg)
        anr.gemm_i8(a, w, sa, sw, d)
    return run, (dx, dg, d)


def test_threads_with_streams_of_their_own(anr):
    """Calls of several launches on workspaces of their own, two threads sharing a stream among them."""
    shared = torch.cuda.Stream()
    run, outs = jobs(anr)
    run()
    want = [o.clone() for o in outs]
    torch.cuda.synchronize()
    wrong = []

    def work(stream):
        mine = [torch.empty_like(o) for o in want]
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            for _ in range(20):
                run(*mine)
        stream.synchronize()
        if not all(torch.equal(o, v) for o, v in zip(mine, want)):
            wrong.append(1)

    threads = [threading.Thread(target=work, args=(s,)) for s in (shared, shared, torch.cuda.Stream(), torch.cuda.Stream())]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not wrong


def test_two_captured_graphs_do_not_share_a_workspace(anr):
    """Replays of two graphs at once on two streams, with eager calls between."""
    all_jobs = []
    for _ in range(2):
        run, outs = jobs(anr)
        run()
        torch.cuda.synchronize()
        want = [o.clone() for o in outs]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
        all_jobs.append((graph, torch.cuda.Stream(), run, outs, want))
    for _ in range(4):
        for _, _, _, outs, _ in all_jobs:
            [o.zero_() for o in outs]
        torch.cuda.synchronize()
        for graph, stream, *_ in all_jobs:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for _, _, run, outs, want in all_jobs:
            assert all(torch.equal(o, w) for o, w in zip(outs, want))
            run()
