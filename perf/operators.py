"""Timed cases of the operators of a transformer block on images, video and tokens: group norm with an activation (channels
last), rotary positions with several axes, and the gated feed-forward block, each forward and backward.

`run` computes them in plain torch operations in 32 bits (angles in 64), or, where `own` is true, makes the calls of the public
binding.  Outputs are tensors that the caller holds already, as everywhere in that binding.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-5

_binding = None


def _anr():
    global _binding
    if _binding is None:
        from paper_2006_06762_amd import binding
        _binding = binding
    return _binding


# ------------------------------------------------------------------ cases
def _norm(direction, N, C, H, W, groups, act, dtype):
    return {"op": "group_norm", "direction": direction, "N": N, "C": C, "H": H, "W": W, "groups": groups, "act": act, "dtype": dtype}


def _rotary(B, S, H, Hk, D, sections, pairing, far, inverse, dtype):
    case = {"op": "rotary", "B": B, "S": S, "H": H, "Hk": Hk, "D": D, "axes": len(sections), "pairing": pairing, "far": far, "inverse": inverse, "dtype": dtype}
    return dict(case, **{"section%d" % i: s for i, s in enumerate(sections)})


def _ff(direction, T, C, F, act, dtype, save=False):
    return {"op": "gated_ff", "direction": direction, "T": T, "C": C, "F": F, "act": act, "dtype": dtype, "save": save}


def listed():
    return [
        # The smallest norm: one image, the last and smallest map of an image network, float32. Latency of one call.
        dict(_norm("forward", 1, 512, 7, 7, 32, "none", "f32"), name="norm_f32_small"),
        # The block norm of an image generator at full resolution, its largest map: one pass over 134 MB.
        dict(_norm("forward", 8, 512, 128, 128, 32, "silu", "bf16"), name="norm_bf16_large"),
        # A training batch's backward pass on the middle maps, float32.
        dict(_norm("backward", 16, 256, 28, 28, 32, "gelu", "f32"), name="norm_f32_backward"),
        # The same in 16 bits on large maps of odd extents, ten channels a group: groups that are no whole 16-byte units.
        dict(_norm("backward", 4, 320, 95, 63, 32, "silu", "bf16"), name="norm_bf16_backward_ragged"),
        # One new token for each of 32 sequences far into a video, query heads that share key heads.
        dict(_rotary(32, 1, 32, 8, 128, (16, 24, 24), "halves", 100000, False, "bf16"), name="rotary_bf16_decode"),
        # Queries and keys of the attention-score benchmark (16 x 128 x 12 x 64), rows and columns of a picture, in the
        # backward pass, float32.
        dict(_rotary(16, 128, 12, 12, 64, (16, 16), "section_halves", 0, True, "f32"), name="rotary_f32_backward"),
        # A clip's tokens at once: the largest, with an odd count of tokens and dimensions that do not turn.
        dict(_rotary(2, 16001, 24, 24, 128, (8, 28, 24), "adjacent", 1000, False, "bf16"), name="rotary_bf16_video"),
        # One token through the block, as a chat's answer has it: bound by reading the weights once.
        dict(_ff("forward", 1, 2048, 5632, "silu", "bf16"), name="ff_bf16_one_token"),
        # A float32 block with the hidden size of the score benchmark (12 heads of 64), pre-activations kept for training.
        dict(_ff("forward", 2048, 768, 2048, "gelu", "f32", True), name="ff_f32_train"),
        # The prompts of a serving batch through a wide layer: the largest products.
        dict(_ff("forward", 8192, 4096, 11264, "silu", "bf16"), name="ff_bf16_prompts"),
        # Backward pass of a training step in 16 bits.
        dict(_ff("backward", 4096, 1024, 2816, "silu", "bf16"), name="ff_bf16_backward"),
        # Backward pass on sizes that are no multiple of anything, float32.
        dict(_ff("backward", 777, 515, 1363, "gelu_tanh", "f32"), name="ff_f32_backward_ragged"),
    ]


_LARGEST_FF = 8192 * 4096 * 11264


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.randrange(5)
    dtype = rng.choice(("f32", "f16", "bf16"))
    if kind < 2:
        while True:
            groups, per = rng.choice((1, 8, 16, 32, 32, 32)), rng.choice((2, 3, 4, 5, 8, 10, 12, 16, 20, 40))
            N, H, W = _log(rng, 1, 16), _log(rng, 4, 128), _log(rng, 4, 128)
            if N * H * W * groups * per <= (1 << 26) * (2 if _BYTES[dtype] == 2 else 1) // 3:
                break
        # (no backward pass through a ReLU: its slope jumps where the last bit of the norm decides)
        acts = ("none", "silu", "gelu", "relu")[:3 if kind else 4]
        return _norm(("forward", "backward")[kind], N, groups * per, H, W, groups, rng.choice(acts), dtype)
    if kind == 2:
        while True:
            B, S, Hk, D = _log(rng, 1, 64), _log(rng, 1, 16384), rng.randint(1, 16), rng.choice((32, 64, 72, 80, 96, 128, 128, 256))
            H = Hk * rng.choice((1, 1, 2, 4, 8))
            if H <= 64 and B * S * (H + Hk) * D <= 1 << 26:
                break
        axes, pairs = rng.randint(1, 3), D // 2 if rng.random() < 0.7 else D // 4
        cuts = sorted(rng.randint(0, pairs) for _ in range(axes - 1))
        sections = [b - a for a, b in zip([0] + cuts, cuts + [pairs])]
        return _rotary(B, S, H, Hk, D, sections, rng.choice(("halves", "adjacent", "section_halves")), rng.choice((0, 1000, 1000000)), rng.random() < 0.4, dtype)
    direction = ("forward", "backward")[kind - 3]
    cost = (2 if direction == "backward" else 1) * (8 if dtype == "f32" else 1)
    while True:
        T, C, F = _log(rng, 1, 8192), _log(rng, 64, 4096), _log(rng, 128, 11264)
        if rng.random() < 0.75:                      # most widths are whole 16-byte units, as layers have them
            C, F = (C + 15) // 16 * 16, (F + 15) // 16 * 16
        if cost * T * C * F <= _LARGEST_FF:
            break
    return _ff(direction, T, C, F, rng.choice(("silu", "gelu", "gelu_tanh", "relu")), dtype, direction == "forward" and rng.random() < 0.5)


def work(case):
    es = _BYTES[case["dtype"]]
    if case["op"] == "group_norm":
        n = case["N"] * case["C"] * case["H"] * case["W"]
        small = 8 * case["N"] * case["groups"] + 2 * case["C"] * es
        if case["direction"] == "forward":
            return {"bytes": 2 * n * es + small, "flops": 8 * n}
        return {"bytes": 3 * n * es + small + 2 * case["C"] * es, "flops": 16 * n}
    if case["op"] == "rotary":
        n, pairs = case["B"] * case["S"] * (case["H"] + case["Hk"]) * case["D"], sum(_sections(case))
        return {"bytes": 2 * n * es + 8 * case["axes"] * case["B"] * case["S"] + 4 * pairs, "flops": 6 * case["B"] * case["S"] * (case["H"] + case["Hk"]) * pairs}
    T, C, F = case["T"], case["C"], case["F"]
    if case["direction"] == "forward":
        return {"bytes": es * (2 * T * C + 3 * C * F + (2 * T * F if case["save"] else 0)), "flops": 6 * T * C * F}
    return {"bytes": es * (3 * T * C + 2 * T * F + 6 * C * F), "flops": 12 * T * C * F}


# ------------------------------------------------------------------ inputs
def _sections(case):
    return tuple(case["section%d" % i] for i in range(case["axes"]))


def _pairs(case):
    """The two dimensions that each pair turns."""
    sections, pairing = _sections(case), case["pairing"]
    n = sum(sections)
    if pairing == "adjacent":
        return [2 * i for i in range(n)], [2 * i + 1 for i in range(n)]
    if pairing == "halves":
        return list(range(n)), [n + i for i in range(n)]
    first, at = [], 0
    for s in sections:
        first += [2 * at + i for i in range(s)]
        at += s
    return first, [f + s for f, s in zip(first, [s for s in sections for _ in range(s)])]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = _TYPES[case["dtype"]]

    def normal(*shape, scale=1.0, shift=0.0):
        return torch.randn(shape, generator=g, device="cuda").mul_(scale).add_(shift).to(t)

    if case["op"] == "group_norm":
        N, C, H, W, groups = (case[k] for k in ("N", "C", "H", "W", "groups"))
        # channels have means and spreads of their own, as behind a convolution with a bias
        spread = torch.rand(C, generator=g, device="cuda") + 0.5
        offset = torch.randn(C, generator=g, device="cuda")
        image = lambda v: v.to(t).permute(0, 3, 1, 2)  # noqa: E731
        x = image(torch.randn(N, H, W, C, generator=g, device="cuda").mul_(spread).add_(offset))
        s = {"case": case, "x": x, "gamma": normal(C, scale=0.2, shift=1.0), "beta": normal(C, scale=0.2)}
        if case["direction"] == "forward":
            s |= {"y": torch.empty_like(x), "mean": torch.empty(N, groups, device="cuda"), "rstd": torch.empty(N, groups, device="cuda")}
        else:
            s["dy"] = image(torch.randn(N, H, W, C, generator=g, device="cuda"))
            rows = x.permute(0, 2, 3, 1).reshape(N, H * W, groups, C // groups)
            mean = torch.stack([r.double().mean((0, 2)) for r in rows])
            var = torch.stack([(r.double() - m[None, :, None]).square().mean((0, 2)) for r, m in zip(rows, mean)])
            s |= {"mean": mean.float(), "rstd": (var + EPS).rsqrt().float()}
            s |= {"dx": torch.empty_like(x), "dgamma": torch.empty_like(s["gamma"]), "dbeta": torch.empty_like(s["beta"])}
        return s
    if case["op"] == "rotary":
        B, S, H, Hk, D, axes = (case[k] for k in ("B", "S", "H", "Hk", "D", "axes"))
        sections = _sections(case)
        pairs = sum(sections)
        # tokens of a clip of square pictures, line by line, behind a text of its own length in each sequence
        edge = max(1, int(round(S ** (1 / max(2, axes)))))
        at = torch.arange(S, device="cuda")
        grid = [at // (edge * edge), at // edge % edge, at % edge][3 - axes:]
        start = torch.randint(0, case["far"] + 1, (B, 1), generator=g, device="cuda")
        positions = torch.stack([a[None, :] + start for a in grid])
        # one run of frequencies over all pairs, or one for each axis where its dimensions are a block of their own
        if case["pairing"] == "section_halves":
            freq = torch.cat([10000.0 ** -(torch.arange(n, dtype=torch.float64) / max(1, n)) for n in sections])
        else:
            freq = 10000.0 ** -(torch.arange(pairs, dtype=torch.float64) / max(1, pairs))
        first, second = _pairs(case)
        q, k = normal(B, S, H, D), normal(B, S, Hk, D)
        of = [a for a, n in enumerate(sections) for _ in range(n)]
        return {"case": case, "q": q, "k": k, "positions": positions, "inv_freq": freq.float().cuda(), "sections": sections, "first": torch.tensor(first, device="cuda"),
                "second": torch.tensor(second, device="cuda"), "axis": torch.tensor(of, device="cuda"), "q_out": torch.empty_like(q), "k_out": torch.empty_like(k)}
    T, C, F = case["T"], case["C"], case["F"]
    s = {"case": case, "x": normal(T, C), "w_gate": normal(F, C, scale=C ** -0.5), "w_up": normal(F, C, scale=C ** -0.5), "w_down": normal(C, F, scale=F ** -0.5)}
    if case["direction"] == "forward":
        s |= {"y": torch.empty_like(s["x"])}
        s |= {k: torch.empty(T, F, dtype=t, device="cuda") if case["save"] else None for k in ("gate", "up")}
    else:
        # what a forward pass left: products of these inputs, rounded once
        s |= {"dy": normal(T, C), "gate": (s["x"].float() @ s["w_gate"].float().t()).to(t), "up": (s["x"].float() @ s["w_up"].float().t()).to(t)}
        s |= {"d" + k: torch.empty_like(s[k]) for k in ("x", "w_gate", "w_up", "w_down")}
    return s


# ------------------------------------------------------------------ the operators
def _act(name, z):
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    return z


def _act_slope(name, z):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def _plain_norm(s, case):
    N, C, H, W, groups = (case[k] for k in ("N", "C", "H", "W", "groups"))
    t = s["x"].dtype
    rows = s["x"].permute(0, 2, 3, 1).reshape(N, H * W, groups, C // groups).float()
    gamma, beta = s["gamma"].float().view(groups, -1), s["beta"].float().view(groups, -1)
    back = lambda v: v.to(t).reshape(N, H, W, C).permute(0, 3, 1, 2)  # noqa: E731
    if case["direction"] == "forward":
        mean = rows.mean((1, 3), keepdim=True)
        centred = rows - mean
        rstd = (centred.square().mean((1, 3), keepdim=True) + EPS).rsqrt()
        return {"y": back(_act(case["act"], centred * rstd * gamma + beta)), "mean": mean.view(N, groups), "rstd": rstd.view(N, groups)}
    rstd = s["rstd"].view(N, 1, groups, 1)
    hat = (rows - s["mean"].view(N, 1, groups, 1)) * rstd
    dz = s["dy"].permute(0, 2, 3, 1).reshape(N, H * W, groups, C // groups).float() * _act_slope(case["act"], hat * gamma + beta)
    dhat = dz * gamma
    dx = rstd * (dhat - dhat.mean((1, 3), keepdim=True) - hat * (dhat * hat).mean((1, 3), keepdim=True))
    return {"dx": back(dx), "dgamma": (dz * hat).sum((0, 1)).view(C).to(t), "dbeta": dz.sum((0, 1)).view(C).to(t)}


def _plain_rotary(s, case):
    angle = s["positions"][s["axis"]].permute(1, 2, 0).double() * s["inv_freq"].double()
    cos, sin = angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]
    if case["inverse"]:
        sin = -sin

    def turn(x):
        out = x.float()
        u, v = out[..., s["first"]], out[..., s["second"]]
        out = out.clone()
        out[..., s["first"]] = u * cos - v * sin
        out[..., s["second"]] = u * sin + v * cos
        return out.to(x.dtype)

    return {"q": turn(s["q"]), "k": turn(s["k"])}


def _plain_ff(s, case):
    x, wg, wu, wd, t = s["x"].float(), s["w_gate"].float(), s["w_up"].float(), s["w_down"].float(), s["x"].dtype
    if case["direction"] == "forward":
        gate, up = x @ wg.t(), x @ wu.t()
        out = {"y": ((_act(case["act"], gate) * up) @ wd.t()).to(t)}
        return out | {"gate": gate.to(t), "up": up.to(t)} if case["save"] else out
    gate, up, dy = s["gate"].float(), s["up"].float(), s["dy"].float()
    a, dh = _act(case["act"], gate), dy @ wd
    dgate, dup = dh * up * _act_slope(case["act"], gate), dh * a
    return {"dx": (dgate @ wg + dup @ wu).to(t), "dw_gate": (dgate.t() @ x).to(t), "dw_up": (dup.t() @ x).to(t), "dw_down": (dy.t() @ (a * up)).to(t)}


def run(s):
    case = s["case"]
    if not own:
        return {"group_norm": _plain_norm, "rotary": _plain_rotary, "gated_ff": _plain_ff}[case["op"]](s, case)
    anr = _anr()
    if case["op"] == "rotary":
        anr.rotary(s["q"], s["k"], s["positions"], s["inv_freq"], s["q_out"], s["k_out"], s["sections"],
                   getattr(anr, "ANR_ROTARY_" + case["pairing"].upper()), case["inverse"])
        return {"q": s["q_out"], "k": s["k_out"]}
    act = getattr(anr, "ANR_ACT_" + case["act"].upper())
    if case["op"] == "group_norm":
        if case["direction"] == "forward":
            anr.group_norm(s["x"], case["groups"], s["y"], s["gamma"], s["beta"], EPS, act, s["mean"], s["rstd"])
            return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
        anr.group_norm_backward(s["dy"], s["x"], case["groups"], s["gamma"], s["beta"], s["mean"], s["rstd"], s["dx"], s["dgamma"], s["dbeta"], act)
        return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    if case["direction"] == "forward":
        anr.gated_ff(s["x"], s["w_gate"], s["w_up"], s["w_down"], s["y"], act, s["gate"], s["up"])
        return {"y": s["y"], "gate": s["gate"], "up": s["up"]} if case["save"] else {"y": s["y"]}
    anr.gated_ff_backward(s["dy"], s["x"], s["w_gate"], s["w_up"], s["w_down"], s["gate"], s["up"], s["dx"], s["dw_gate"], s["dw_up"], s["dw_down"], act)
    return {"dx": s["dx"], "dw_gate": s["dw_gate"], "dw_up": s["dw_up"], "dw_down": s["dw_down"]}


# ------------------------------------------------------------------ the definitions, in 64 bits
def _value_and_slope(name, z):
    """act(z) and its derivative, the derivative by automatic differentiation of the definition."""
    with torch.enable_grad():
        z = z.detach().requires_grad_()
        if name == "relu":
            a = z.clamp(min=0)
        elif name == "silu":
            a = z * torch.sigmoid(z)
        elif name == "gelu":
            a = z * torch.special.ndtr(z)
        elif name == "gelu_tanh":
            a = z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
        else:
            a = z * 1.0
        slope, = torch.autograd.grad(a.sum(), z)
    return a.detach(), slope


def exact(case, seed):
    s = prepare(case, seed)
    t = torch.float64
    if case["op"] == "group_norm":
        N, C, groups = case["N"], case["C"], case["groups"]
        per = C // groups
        x = s["x"]
        gamma, beta = s["gamma"].to(t)[:, None, None], s["beta"].to(t)[:, None, None]
        spread = lambda v: v.repeat_interleave(per)[:, None, None]  # noqa: E731
        if case["direction"] == "forward":
            y, means, rstds = torch.empty(x.shape, dtype=t, device=x.device, memory_format=torch.channels_last), [], []
            for i in range(N):
                image = x[i].to(t)
                flat = image.reshape(groups, -1)
                mean = flat.mean(1)
                rstd = 1 / torch.sqrt(flat.var(1, unbiased=False) + EPS)
                y[i] = _value_and_slope(case["act"], (image - spread(mean)) * spread(rstd) * gamma + beta)[0]
                means.append(mean)
                rstds.append(rstd)
            return {"y": y, "mean": torch.stack(means), "rstd": torch.stack(rstds)}
        dx, dgamma, dbeta = torch.empty(x.shape, dtype=t, device=x.device, memory_format=torch.channels_last), 0, 0
        for i in range(N):
            mean, rstd = spread(s["mean"][i].to(t)), spread(s["rstd"][i].to(t))
            hat = (x[i].to(t) - mean) * rstd
            dz = s["dy"][i].to(t) * _value_and_slope(case["act"], gamma * hat + beta)[1]
            dgamma, dbeta = dgamma + (dz * hat).sum((1, 2)), dbeta + dz.sum((1, 2))
            dhat = gamma * dz
            part = lambda v: spread(v.reshape(groups, -1).mean(1))  # noqa: E731
            dx[i] = (dhat - part(dhat) - part(dhat * hat) * hat) * rstd
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    if case["op"] == "rotary":
        cuts = [s["positions"][a].to(t)[..., None] * f.to(t) for a, f in enumerate(s["inv_freq"].split(list(s["sections"])))]
        angle = torch.cat(cuts, -1)
        unit = torch.polar(torch.ones_like(angle), -angle if case["inverse"] else angle)[:, :, None]
        first, second = _pairs(case)
        out = {}
        for name in ("q", "k"):
            x = s[name].to(t)
            z = torch.complex(x[..., first], x[..., second]) * unit
            y = x.clone()
            y[..., first], y[..., second] = z.real, z.imag
            out[name] = y
        return out
    x, wg, wu, wd = (s[k].to(t) for k in ("x", "w_gate", "w_up", "w_down"))
    if case["direction"] == "forward":
        gate, up = torch.mm(x, wg.t().contiguous()), torch.mm(x, wu.t().contiguous())
        out = {"y": torch.mm(_value_and_slope(case["act"], gate)[0].mul_(up), wd.t().contiguous())}
        return dict(out, gate=gate, up=up) if case["save"] else out
    gate, up, dy = (s[k].to(t) for k in ("gate", "up", "dy"))
    a, slope = _value_and_slope(case["act"], gate)
    dh = torch.mm(dy, wd)
    dgate, dup = dh * slope * up, dh * a
    return {"dx": torch.mm(torch.cat((dgate, dup), 1), torch.cat((wg, wu))), "dw_gate": torch.mm(dgate.t().contiguous(), x), "dw_up": torch.mm(dup.t().contiguous(), x),
            "dw_down": torch.mm(dy.t().contiguous(), a * up)}
