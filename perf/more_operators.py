"""Timed cases of the operators around a transformer block's products in 8 bits: root-mean-square norm with the residual's
addition, forward and backward and with an output in 8 bits, rows of values in 8 bits with a scale each, and the product of 8-bit
integers with scales for tokens and channels.

`run` computes them in plain torch operations in 32 bits, or, where `own` is true, makes the calls of the public binding.  Outputs
are tensors that the caller holds already, as everywhere in that binding; what is held in 8 bits is read back as 16-bit values.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-6

_binding = None


def _anr():
    global _binding
    if _binding is None:
        from paper_2006_06762_amd import binding
        _binding = binding
    return _binding


# ------------------------------------------------------------------ cases
def _norm(direction, T, C, residual, dtype, param):
    """direction: forward, backward, or quantized (forward with an output in 8 bits)."""
    return {"op": "rms_norm", "direction": direction, "T": T, "C": C, "residual": residual, "dtype": dtype, "param": param}


def _quantize(T, C, act, gated, dtype):
    return {"op": "quantize", "T": T, "C": C, "act": act, "gated": gated, "dtype": dtype}


def _product(T, K, N, bias, dtype):
    return {"op": "product", "T": T, "K": K, "N": N, "bias": bias, "dtype": dtype}


def _norm_product(T, K, N, dtype):
    return {"op": "norm_product", "T": T, "K": K, "N": N, "dtype": dtype}


def listed():
    return [
        # One new token's norm behind an attention block: the smallest, latency of one call.
        dict(_norm("forward", 1, 2048, True, "bf16", "bf16"), name="norm_bf16_one_token"),
        # Float32 training with the hidden size of the score benchmark (12 heads of 64).
        dict(_norm("forward", 2048, 768, False, "f32", "f32"), name="norm_f32_train"),
        # The prompts of a serving batch through a wide layer: one pass over four matrices of 134 MB.
        dict(_norm("forward", 16384, 4096, True, "bf16", "bf16"), name="norm_bf16_prompts"),
        # Backward pass of a training step in 16 bits, with the gradient of the residual stream; float32 parameters.
        dict(_norm("backward", 8192, 4096, True, "bf16", "f32"), name="norm_bf16_backward"),
        # Float32 backward pass on sizes that are no multiple of anything.
        dict(_norm("backward", 3001, 1363, False, "f32", "f32"), name="norm_f32_backward_ragged"),
        # The norm in front of an 8-bit product, for a serving batch's prompts.
        dict(_norm("quantized", 8192, 4096, True, "bf16", "bf16"), name="norm_8bit_prompts"),
        # One token from the residual stream through the norm and the gate's and up's weights in 8 bits: bound by reading them.
        dict(_norm_product(1, 2048, 11264, "bf16"), name="norm_product_one_token"),
        # Between the products of a gated feed-forward block: gate and up are the halves of the first one's result.
        dict(_quantize(8192, 11264, "silu", True, "bf16"), name="quantize_gated_prompts"),
        # Float32 weights to 8 bits, a scale for each output channel; rows that are no whole 16-byte units.
        dict(_quantize(2777, 1001, "none", False, "f32"), name="quantize_weights_ragged"),
        # One token each of 32 sequences.
        dict(_product(32, 4096, 11264, False, "bf16"), name="product_decode_batch"),
        # The prompts of a serving batch through a wide layer: the largest product.
        dict(_product(8192, 4096, 11264, False, "bf16"), name="product_prompts"),
        # Sizes that are no multiple of anything, float32 results with a bias.
        dict(_product(777, 515, 1363, True, "f32"), name="product_f32_ragged"),
    ]


_MOST_PRODUCTS = 8192 * 4096 * 11264
_MOST_BYTES = 4 * 2 * 16384 * 4096


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.randrange(6)
    dtype = rng.choice(("f32", "f16", "bf16"))
    units = rng.random() < 0.7               # most widths are whole 16-byte units, as layers have them
    whole = lambda n: (n + 15) // 16 * 16 if units else n  # noqa: E731
    if kind < 3:
        direction = ("forward", "backward", "quantized")[kind]
        while True:
            case = _norm(direction, _log(rng, 1, 32768), whole(_log(rng, 64, 16384)), rng.random() < 0.6, dtype, rng.choice(("f32", dtype)))
            if work(case)["bytes"] <= _MOST_BYTES:
                return case
    if kind == 3:
        while True:
            gated = rng.random() < 0.6
            act = rng.choice(("silu", "gelu", "gelu_tanh", "relu")) if gated else rng.choice(("none", "none", "gelu", "relu"))
            case = _quantize(_log(rng, 1, 32768), whole(_log(rng, 64, 16384)), act, gated, dtype)
            if work(case)["bytes"] <= _MOST_BYTES:
                return case
    while True:
        T, K, N = _log(rng, 1, 16384), whole(_log(rng, 64, 16384)), whole(_log(rng, 64, 16384))
        if T * K * N <= _MOST_PRODUCTS and _BYTES[dtype] * T * N <= _MOST_BYTES:
            break
    if kind == 4 and dtype != "f32":
        return _norm_product(T, K, N, dtype)
    return _product(T, K, N, rng.random() < 0.3, dtype)


def work(case):
    es, T = _BYTES[case["dtype"]], case["T"]
    if case["op"] == "rms_norm":
        n = T * case["C"]
        parameters = case["C"] * _BYTES[case["param"]]
        if case["direction"] == "backward":
            return {"bytes": (4 if case["residual"] else 3) * n * es + 2 * parameters + 4 * T, "flops": 10 * n}
        held = (3 if case["residual"] else 1) * n * es + parameters + 4 * T
        return {"bytes": held + (n * es if case["direction"] == "forward" else 3 * n), "flops": 6 * n}
    if case["op"] == "quantize":
        n = T * case["C"]
        return {"bytes": n * es * (2 if case["gated"] else 1) + 3 * n + 4 * T, "flops": 6 * n}
    K, N = case["K"], case["N"]
    if case["op"] == "norm_product":
        return {"bytes": 3 * T * K * es + K * es + N * K + 4 * N + T * N * es, "flops": 2 * T * K * N + 6 * T * K}
    return {"bytes": T * K + N * K + 4 * (T + N) + T * N * es + (4 * N if case["bias"] else 0), "flops": 2 * T * K * N}


# ------------------------------------------------------------------ inputs
def _rows_in_8_bits(v):
    largest = v.abs().amax(1, keepdim=True)
    return torch.round(v * (127 / largest)).to(torch.int8), (largest / 127).flatten()


def _read_back(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float16


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t, T = _TYPES[case["dtype"]], case["T"]

    def normal(*shape, scale=1.0, shift=0.0, dtype=t):
        return torch.randn(shape, generator=g, device="cuda").mul_(scale).add_(shift).to(dtype)

    def stream(C):
        # tokens of different size, and one channel in a hundred that is much larger than the others
        channel = torch.where(torch.rand(C, generator=g, device="cuda") < 0.01, 8.0, 1.0)
        return torch.randn(T, C, generator=g, device="cuda").mul_(channel).mul_(torch.rand(T, 1, generator=g, device="cuda") + 0.5).to(t)

    def weights(N, K):
        return _rows_in_8_bits(torch.randn(N, K, generator=g, device="cuda").mul_(K ** -0.5))

    empty = lambda *shape, dtype=t: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    s = {"case": case}
    if case["op"] == "rms_norm":
        C, p = case["C"], _TYPES[case["param"]]
        s |= {"x": stream(C), "gamma": normal(C, scale=0.2, shift=1.0, dtype=p)}
        if case["direction"] == "backward":
            s |= {"dy": normal(T, C), "dh": normal(T, C) if case["residual"] else None}
            # what a forward pass left
            s["rstd"] = torch.cat([(r.double().square().mean(1) + EPS).rsqrt().float() for r in s["x"].split(4096)])
            return s | {"dx": empty(T, C), "dgamma": empty(C, dtype=p)}
        s |= {"residual": normal(T, C), "h": empty(T, C)} if case["residual"] else {"residual": None, "h": None}
        if case["direction"] == "forward":
            return s | {"y": empty(T, C), "rstd": empty(T, dtype=torch.float32)}
        return s | {"q": empty(T, C, dtype=torch.int8), "scale": empty(T, dtype=torch.float32), "y": empty(T, C, dtype=_read_back(case))}
    if case["op"] == "quantize":
        C = case["C"]
        both = normal(T, 2 * C if case["gated"] else C)
        s |= {"x": both[:, :C], "up": both[:, C:] if case["gated"] else None}
        return s | {"q": empty(T, C, dtype=torch.int8), "scale": empty(T, dtype=torch.float32), "y": empty(T, C, dtype=_read_back(case))}
    K, N = case["K"], case["N"]
    s |= dict(zip(("w", "w_scale"), weights(N, K)), d=empty(T, N))
    if case["op"] == "norm_product":
        s |= {"x": stream(K), "residual": normal(T, K), "h": empty(T, K), "gamma": normal(K, scale=0.2, shift=1.0)}
        return s | {"q": empty(T, K, dtype=torch.int8), "scale": empty(T, dtype=torch.float32)}
    s |= dict(zip(("a", "a_scale"), _rows_in_8_bits(torch.randn(T, K, generator=g, device="cuda"))))
    return s | {"bias": normal(N, dtype=torch.float32) if case["bias"] else None}


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


def _plain_norm(s):
    """h, the normed rows and their rstd, all in 32 bits."""
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    rstd = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
    return h, h * rstd * s["gamma"].float(), rstd


def _plain_8_bits(v):
    largest = v.abs().amax(1, keepdim=True)
    return torch.round(v * (127 / largest)), largest / 127


def _plain(s, case):
    op, t = case["op"], _TYPES[case["dtype"]]
    if op == "rms_norm" and case["direction"] == "backward":
        hat, rstd, dy = s["x"].float() * s["rstd"][:, None], s["rstd"][:, None], s["dy"].float()
        dhat = dy * s["gamma"].float()
        dx = rstd * (dhat - hat * (dhat * hat).mean(1, keepdim=True))
        if s["dh"] is not None:
            dx = dx + s["dh"].float()
        return {"dx": dx.to(t), "dgamma": (dy * hat).sum(0).to(s["dgamma"].dtype)}
    if op == "rms_norm":
        h, y, rstd = _plain_norm(s)
        out = {} if s["h"] is None else {"h": h.to(t)}
        if case["direction"] == "forward":
            return out | {"y": y.to(t), "rstd": rstd.flatten()}
        q, scale = _plain_8_bits(y)
        return out | {"y": (q * scale).to(_read_back(case)), "scale": scale.flatten()}
    if op == "quantize":
        v = _act(case["act"], s["x"].float())
        if s["up"] is not None:
            v = v * s["up"].float()
        q, scale = _plain_8_bits(v)
        return {"y": (q * scale).to(_read_back(case)), "scale": scale.flatten()}
    if op == "norm_product":
        h, y, _ = _plain_norm(s)
        q, scale = _plain_8_bits(y)
        return {"h": h.to(t), "d": (q @ s["w"].float().t() * scale * s["w_scale"]).to(t)}
    d = s["a"].float() @ s["w"].float().t() * s["a_scale"][:, None] * s["w_scale"]
    if s["bias"] is not None:
        d = d + s["bias"]
    return {"d": d.to(t)}


def run(s):
    case = s["case"]
    if not own:
        return _plain(s, case)
    anr = _anr()
    if case["op"] == "rms_norm":
        if case["direction"] == "backward":
            anr.rms_norm_backward(s["dy"], s["x"], s["gamma"], s["rstd"], s["dx"], s["dgamma"], s["dh"])
            return {"dx": s["dx"], "dgamma": s["dgamma"]}
        out = {} if s["h"] is None else {"h": s["h"]}
        if case["direction"] == "forward":
            anr.rms_norm(s["x"], s["y"], s["gamma"], EPS, s["residual"], s["h"], s["rstd"])
            return out | {"y": s["y"], "rstd": s["rstd"]}
        anr.rms_norm_q8(s["x"], s["q"], s["scale"], s["gamma"], EPS, s["residual"], s["h"])
        anr.dequantize_rows(s["q"], s["scale"], s["y"])
        return out | {"y": s["y"], "scale": s["scale"]}
    if case["op"] == "quantize":
        anr.quantize_rows(s["x"], s["q"], s["scale"], getattr(anr, "ANR_ACT_" + case["act"].upper()), s["up"])
        anr.dequantize_rows(s["q"], s["scale"], s["y"])
        return {"y": s["y"], "scale": s["scale"]}
    if case["op"] == "norm_product":
        anr.rms_norm_q8(s["x"], s["q"], s["scale"], s["gamma"], EPS, s["residual"], s["h"])
        anr.gemm_i8(s["q"], s["w"], s["scale"], s["w_scale"], s["d"])
        return {"h": s["h"], "d": s["d"]}
    anr.gemm_i8(s["a"], s["w"], s["a_scale"], s["w_scale"], s["d"], s["bias"])
    return {"d": s["d"]}


# ------------------------------------------------------------------ the definitions, in 64 bits
def _value(name, z):
    if name == "relu":
        return z.clamp(min=0)
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu":
        return z * torch.special.ndtr(z)
    if name == "gelu_tanh":
        return z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
    return z


def _steps(v):
    """The nearest whole steps, and the steps: the largest of a row is 127 of them."""
    step = v.abs().max(dim=1, keepdim=True).values / 127
    return torch.div(v, step).round(), step


def exact(case, seed):
    s = prepare(case, seed)
    wide = lambda k: s[k].to(torch.float64)  # noqa: E731
    op = case["op"]
    if op == "rms_norm" and case["direction"] == "backward":
        x, dy, gamma, rstd = wide("x"), wide("dy"), wide("gamma"), wide("rstd").unsqueeze(1)
        C = x.shape[1]
        along = torch.linalg.vecdot(dy * gamma, x).unsqueeze(1)
        dx = dy * gamma * rstd - x * along * rstd ** 3 / C
        if s["dh"] is not None:
            dx += wide("dh")
        return {"dx": dx, "dgamma": torch.mv((dy * x).t(), wide("rstd"))}
    if op in ("rms_norm", "norm_product"):
        h = wide("x")
        if s["residual"] is not None:
            h += wide("residual")
        rstd = 1 / torch.sqrt(torch.linalg.vecdot(h, h) / h.shape[1] + EPS)
        y = h * (rstd[:, None] * wide("gamma"))
        out = {} if s["h"] is None else {"h": h}
        if op == "rms_norm" and case["direction"] == "forward":
            return dict(out, y=y, rstd=rstd)
        q, step = _steps(y)
        if op == "rms_norm":
            return dict(out, y=q * step, scale=step[:, 0])
        return dict(out, d=torch.mm(q * step, (wide("w") * wide("w_scale")[:, None]).t().contiguous()))
    if op == "quantize":
        v = _value(case["act"], wide("x"))
        if s["up"] is not None:
            v *= wide("up")
        q, step = _steps(v)
        return {"y": q * step, "scale": step[:, 0]}
    d = torch.mm(wide("a"), wide("w").t().contiguous())
    d = d * torch.outer(wide("a_scale"), wide("w_scale"))
    return {"d": d if s["bias"] is None else d + wide("bias")}
