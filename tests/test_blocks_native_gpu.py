"""The extension module's group norm, rotary positions and gated feed-forward block against the Python functions it stands
before: the same results for every way to pass the arguments, and the same errors; calls of threads, on streams and in captures."""
import threading

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

NAMES = ["group_norm", "group_norm_backward", "rotary", "gated_ff", "gated_ff_backward"]


@pytest.fixture(scope="module")
def anr():
    from paper_2006_06762_amd import binding
    return binding


def rand(*shape, t=torch.float32):
    return (torch.rand(shape, device="cuda") - 0.5).to(t)


def image(N, C, H, W, t=torch.float32, spare=0):
    return rand(N, H, W, C + spare, t=t)[..., :C].permute(0, 3, 1, 2)


def calls(anr, name):
    """(args, kwargs, outputs) of calls that the extension module takes and of some that go to Python."""
    out = []
    for t in (torch.float32, torch.float16, torch.bfloat16):
        x, y, dy, dx = (image(2, 24, 6, 5, t) for _ in range(4))
        g, b, dg, db = (rand(24, t=t) for _ in range(4))
        mean, rstd = rand(2, 4), rand(2, 4).abs() + 0.5
        rows = [rand(2, 30, 24, t=t).transpose(1, 2) for _ in range(2)]
        wide = [image(2, 24, 6, 5, t, 3) for _ in range(2)]
        if name == "group_norm":
            out += [((x, 4, y), {}, [y]), ((x, 4, y, g, b), {"eps": 1e-3, "act": anr.ANR_ACT_SILU, "mean": mean, "rstd": rstd}, [y, mean, rstd]),
                    ((x, 4, y, None, None, 1, 3, mean, None, None), {}, [y, mean]), ((rows[0], 3), {"y": rows[1], "beta": b.float()}, [rows[1]]),
                    ((wide[0], 8, wide[1], g), {"ws": torch.empty(1 << 16, dtype=torch.uint8, device="cuda")}, [wide[1]])]
        elif name == "group_norm_backward":
            out += [((dy, x, 4, g, b, mean, rstd, dx, dg, db), {}, [dx, dg, db]), ((dy, x, 4, None, None, mean, rstd), {"dx": dx, "act": anr.ANR_ACT_GELU}, [dx]),
                    ((dy, x, 4, g, b, mean, rstd, None, dg), {"dbeta": db, "act": 2}, [dg, db]), ((wide[0], x, 4, g, b, mean, rstd, wide[1]), {}, [wide[1]])]
        elif name == "rotary":
            q, k, qo, ko = rand(2, 7, 4, 32, t=t), rand(2, 7, 2, 32, t=t), rand(2, 7, 4, 32, t=t), rand(2, 7, 2, 32, t=t)
            pos, f = torch.randint(0, 99, (2, 2, 7), device="cuda"), rand(16)
            view = rand(2, 4, 7, 32, t=t).transpose(1, 2)
            out += [((q, k, pos, f, qo, ko, (8, 8)), {}, [qo, ko]), ((q, None, pos[:1], f, qo, None), {"inverse": True}, [qo]),
                    ((q, k, pos[:, 0].int(), f, qo, ko, (4, 12), anr.ANR_ROTARY_ADJACENT, False), {}, [qo, ko]), ((view, k, pos.float(), f, qo, ko), {"sections": [8, 8], "pairing": 2}, [qo, ko]),
                    ((q, k, pos[:, :1].expand(2, 2, 7), f, view, ko, (16, 0)), {}, [view, ko])]
        else:
            big = name == "gated_ff" and t is not torch.float16
            T, C, F = (200, 64, 96) if big else (9, 40, 56)
            x, y, dy, dx = (rand(T, C, t=t) for _ in range(4))
            both = rand(2 * F, C, t=t)
            wd, dwd = rand(C, F, t=t), rand(C, F, t=t)
            wg, wu, dwg, dwu = both[:F], both[F:], rand(F, C, t=t), rand(F, C, t=t)
            gate, up = rand(T, F, t=t), rand(T, F, t=t)
            strided = rand(T, C + 8, t=t)[:, :C]
            if name == "gated_ff":
                out += [((x, wg, wu, wd, y), {}, [y]), ((x, wg, wu, wd), {"y": y, "gate": gate, "up": up, "act": anr.ANR_ACT_GELU}, [y, gate, up]),
                        ((strided, wg, wu, wd, y, 0, None, None, None), {}, [y]), ((x, wg, wu, wd, strided), {"ws": torch.empty(1 << 20, dtype=torch.uint8, device="cuda")}, [strided]),
                        ((x[:1], wg, wu, wd, y[:1]), {}, [y[:1]])]
            else:
                out += [((dy, x, wg, wu, wd, gate, up, dx, dwg, dwu, dwd), {}, [dx, dwg, dwu, dwd]), ((dy, x, wg, wu, wd, gate, up), {"dx": dx, "act": 1}, [dx]),
                        ((dy, x, wg, wu, wd, gate, up, None, None, dwu), {"dw_down": dwd}, [dwu, dwd]), ((strided, x, wg, wu, wd, gate, up, dx, dwg), {}, [dx, dwg])]
    return out


@pytest.mark.parametrize("name", NAMES)
def test_same_results(anr, name):
    for args, kwargs, outs in calls(anr, name):
        for o in outs:
            o.fill_(float("nan"))
        python = getattr(anr, "_" + name)(*args, **kwargs)
        want = [o.clone() for o in outs]
        assert not any(torch.isnan(w).any() for w in want)
        for on in (torch.cuda.current_stream(), torch.cuda.Stream()):
            for o in outs:
                o.fill_(float("nan"))
            on.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(on):
                native = getattr(anr, name)(*args, **kwargs)
            torch.cuda.synchronize()
            assert all(torch.equal(o, w) for o, w in zip(outs, want))
            assert type(native) is type(python)
            assert native is python if not isinstance(python, tuple) else all(a is b for a, b in zip(native, python)) and len(native) == len(python)


def test_same_errors(anr):
    x, q, m = image(2, 16, 4, 4), rand(1, 3, 2, 16), rand(6, 8)
    pos, f, s = torch.zeros(1, 3, dtype=torch.int64, device="cuda"), rand(8), rand(2, 4)
    bad = [("group_norm", (x, 4), {}), ("group_norm", (x, 5, x), {}), ("group_norm", (x.contiguous(), 4, x), {}), ("group_norm", (x, 4, x.half()), {}), ("group_norm", (x, 4, x, 3), {}),
           ("group_norm", (x, 4, x.cpu()), {}), ("group_norm", (x, 4.0, x), {}), ("group_norm", (x, 4, x), {"act": 7}), ("group_norm", (x, 4, x), {"eps": -1.0}), ("group_norm", (x, 4, x), {"mean": s.t()}),
           ("group_norm", (x, 4, x), {"gama": f}), ("group_norm", (x, 4, x), {"gamma": f}), ("group_norm", (m, 4, m), {}), ("group_norm", (x, 1 << 40, x), {}),
           ("group_norm_backward", (x, x, 4, None, None, s, s), {}), ("group_norm_backward", (x, x, 4, None, None, None, s, x), {}), ("group_norm_backward", (x, x[:1], 4, None, None, s, s, x), {}),
           ("rotary", (q, None, pos, f, q), {}), ("rotary", (q, q, pos, f, q, None), {}), ("rotary", (q, None, pos, f, q, None, (4,)), {}), ("rotary", (q, None, pos, f, q, None, (8, 0)), {}),
           ("rotary", (q, None, pos, f, q, None, None, 5), {}), ("rotary", (q, None, pos.short(), f, q, None), {}), ("rotary", (q, None, pos, rand(9), rand(1, 3, 2, 16), None), {}),
           ("rotary", (q, None, pos[:, :2], f, q, None), {}), ("rotary", (q[0], None, pos, f, q[0], None), {}), ("rotary", (q, 3, pos, f, q, 3), {}),
           ("gated_ff", (m, m, m, m), {}), ("gated_ff", (m, m, m, m, m), {}), ("gated_ff", (m, m, m, m.t(), m), {"gate": m}), ("gated_ff", (m, m, m, m.t().contiguous(), m, 17), {}),
           ("gated_ff", (m, m, m[:4], m.t().contiguous(), m), {}), ("gated_ff", (m.double(), m, m, m, m), {}), ("gated_ff", (m, m, m, m.t().contiguous(), m.t()), {}),
           ("gated_ff_backward", (m, m, m, m, m.t().contiguous(), rand(6, 6), rand(6, 6)), {}), ("gated_ff_backward", (m, m, m, m, m.t().contiguous(), None, rand(6, 6), m), {})]
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

    x, y = rand(20, 16), rand(20, 16)
    w = [rand(24, 16), rand(24, 16), rand(16, 24)]
    want = anr._gated_ff(x, *w, y).clone()
    assert torch.equal(anr.gated_ff(x, *(torch.nn.Parameter(v) for v in w), y.zero_()), want)
    assert torch.equal(anr.gated_ff(x.as_subclass(Sub), *w, y.zero_()), want)


def test_threads_with_streams_of_their_own(anr):
    """Calls of several launches on workspaces of their own, two threads sharing a stream among them."""
    shared = torch.cuda.Stream()
    x = image(4, 64, 40, 40, torch.bfloat16)
    a, w = rand(150, 512, t=torch.bfloat16), [rand(256, 512, t=torch.bfloat16), rand(256, 512, t=torch.bfloat16), rand(512, 256, t=torch.bfloat16)]
    norm = anr.group_norm(x, 8, torch.empty_like(x)).clone()
    ff = anr.gated_ff(a, *w, torch.empty_like(a)).clone()
    torch.cuda.synchronize()
    wrong = []

    def work(stream):
        y, b = torch.empty_like(x), torch.empty_like(a)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            for _ in range(20):
                anr.group_norm(x, 8, y)
                anr.gated_ff(a, *w, b)
        stream.synchronize()
        if not (torch.equal(y, norm) and torch.equal(b, ff)):
            wrong.append(1)

    threads = [threading.Thread(target=work, args=(s,)) for s in (shared, shared, torch.cuda.Stream(), torch.cuda.Stream())]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not wrong


def test_two_captured_graphs_do_not_share_a_workspace(anr):
    """Replays of two graphs at once on two streams, with eager calls between."""
    jobs = []
    for i in range(2):
        x, y = image(4, 64, 48, 48, torch.float32), image(4, 64, 48, 48, torch.float32)
        a, w = rand(300, 256, t=torch.bfloat16), [rand(384, 256, t=torch.bfloat16), rand(384, 256, t=torch.bfloat16), rand(256, 384, t=torch.bfloat16)]
        b = torch.empty_like(a)

        def run(x=x, y=y, a=a, w=w, b=b):
            anr.group_norm(x, 8, y, act=anr.ANR_ACT_GELU)
            anr.gated_ff(a, *w, b)
        run()
        torch.cuda.synchronize()
        want = y.clone(), b.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
        jobs.append((graph, torch.cuda.Stream(), y, b, want, run))
    for _ in range(4):
        for graph, stream, y, b, want, run in jobs:
            y.zero_(), b.zero_()
        torch.cuda.synchronize()
        for graph, stream, *_ in jobs:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for graph, stream, y, b, want, run in jobs:
            assert torch.equal(y, want[0]) and torch.equal(b, want[1])
            run()
