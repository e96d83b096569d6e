"""Cases of the 8-bit operators: blocks of 128 values with one power-of-two scale (F8), the product of such operands, the
root-mean-square norm with the residual's addition that produces them, and rotary positions with several axes.

Number format (one block = 128 consecutive values of an item): with a = max |v| = m 2^x, 1 <= m < 2, the scale is 2^(x - 8) for
m <= 1.75 and 2^(x - 7) above, never below 2^-127; each value divided by the scale is rounded to the nearest E4M3 value (ties to
the even mantissa).

`run` computes one pass either in plain torch operations, in 32 bits (`own` false), or through the library's calls.
"""
import math

import torch

own = False

BLOCK = 128
_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- cases --------------------------------------------------------------------------------------------------------

def listed():
    return [
        # rows that end inside a block, fp32 results of another layer
        {"name": "quantize_odd", "op": "quantize", "rows": 777, "k": 1111, "dtype": "f32"},
        # a large layer's activations (or its weights, once)
        {"name": "quantize_large", "op": "quantize", "rows": 16384, "k": 8192, "dtype": "bf16"},
        # the norm in front of a layer at one token
        {"name": "norm_token", "op": "norm", "rows": 1, "k": 8192, "dtype": "bf16", "res": "bf16", "out": "bf16"},
        # a norm without residual over rows that are no multiple of anything, fp32 throughout
        {"name": "norm_odd", "op": "norm", "rows": 777, "k": 1111, "dtype": "f32", "res": "none", "out": "f32"},
        # a prompt's tokens: residual added, normalised, handed on in 8 bits (and read back)
        {"name": "norm_prompt", "op": "norm", "rows": 16384, "k": 8192, "dtype": "bf16", "res": "bf16", "out": "f8"},
        # a dense layer at one token: the weights are read once, nothing is reused
        {"name": "dense_token", "op": "dense", "m": 1, "k": 8192, "o": 8192, "relu": False, "out": "bf16"},
        # a batch of sequences, one token each: the norm and the layer behind it
        {"name": "layer_batch", "op": "layer", "m": 64, "k": 8192, "o": 8192, "relu": False, "out": "bf16"},
        # both operands already in 8 bits, nothing a multiple of anything
        {"name": "product_odd", "op": "product", "m": 301, "k": 1111, "o": 777, "relu": True, "out": "bf16"},
        # the framework's headline product with both operands held in 8 bits
        {"name": "product_4096", "op": "product", "m": 4096, "k": 4096, "o": 4096, "relu": True, "out": "f32"},
        # a prompt's worth of tokens through a large layer
        {"name": "dense_large", "op": "dense", "m": 16384, "k": 8192, "o": 8192, "relu": False, "out": "bf16"},
        # one step of a batch in flight: queries and keys of a fused projection, behind contexts of up to a million tokens
        {"name": "rotate_token", "op": "rotate", "batch": 64, "t": 1, "heads": 40, "rest": 8, "d": 128, "pairs": 64, "axes": 1,
         "adjacent": False, "far": 1 << 20, "dtype": "bf16"},
        # two prompts of text and images: time, height and width
        {"name": "rotate_image", "op": "rotate", "batch": 2, "t": 4099, "heads": 40, "rest": 8, "d": 128, "pairs": 64, "axes": 3,
         "adjacent": False, "far": 32768, "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["quantize", "norm", "norm", "dense", "product", "layer", "rotate", "rotate"])
    if op in ("quantize", "norm"):
        rows = _log(rng, 1, 16384)
        case = {"op": op, "rows": rows, "k": _log(rng, 1, min(16384, 16384 * 8192 // rows)), "dtype": rng.choice(["bf16", "f32"])}
        if op == "norm":
            case.update(res=rng.choice(["none", "bf16", "f32"]), out=rng.choice(["bf16", "f32", "f8"]))
        return case
    if op != "rotate":
        return {"op": op, "m": _log(rng, 1, 16384), "k": _log(rng, 17, 8192), "o": _log(rng, 9, 8192),
                "relu": rng.random() < 0.5, "out": rng.choice(["bf16", "f32"])}
    d = rng.choice([48, 64, 80, 96, 128, 256])
    pairs = rng.choice([d // 2, d // 2, d // 4])
    t = 1 if rng.random() < 0.4 else _log(rng, 1, 8192)
    return {"op": op, "batch": _log(rng, 1, max(1, min(256, 8192 // t))), "t": t, "heads": _log(rng, 1, 64), "rest": rng.choice([0, 1, 8]),
            "d": d, "pairs": pairs, "axes": rng.choice([1, 2, 3, 4]), "adjacent": rng.random() < 0.4, "far": _log(rng, 16, 1 << 20),
            "dtype": rng.choice(["bf16", "bf16", "f32"])}


def _sections(case):
    """Pairs of each axis, one stretch after the other (the first axis has what does not divide)."""
    n, axes = case["pairs"], case["axes"]
    return [n - (axes - 1) * (n // axes)] + [n // axes] * (axes - 1)


# ---- inputs: what a program has in hand ---------------------------------------------------------------------------

_THETA = 500000.0
_EPS = 1e-5


def _device():
    return torch.device("cuda", torch.cuda.current_device())


def _normal(shape, g, std=1.0, dtype=torch.bfloat16):
    return (torch.randn(shape, generator=g, device=g.device) * std).to(dtype)


def _activations(rows, k, g, dtype):
    """N(0,1) with a few channels an order of magnitude larger, as layer inputs have."""
    x = torch.randn((rows, k), generator=g, device=g.device)
    loud = torch.rand((k,), generator=g, device=g.device) < 0.01
    return torch.where(loud, x * 12.0, x).to(dtype)


def _inputs(case, seed):
    """The raw values of a case, made from the seed alone."""
    g = torch.Generator(device=_device()).manual_seed(1000003 * int(seed) + 29)
    op = case["op"]
    if op == "quantize":
        return {"x": _activations(case["rows"], case["k"], g, _DT[case["dtype"]])}
    if op == "rotate":
        b, t = case["batch"], case["t"]
        # positions of each axis: a stretch of consecutive places that ends before `far`
        start = torch.randint(0, case["far"], (case["axes"], b, 1), generator=g, device=g.device)
        step = torch.randint(0, 3, (case["axes"], b, t), generator=g, device=g.device)
        at = (start + step.cumsum(-1)).clamp_max(case["far"]).to(torch.int32)
        return {"qkv": _normal((b, t, case["heads"] + case["rest"], case["d"]), g, 1.0, _DT[case["dtype"]]), "positions": at}
    rows = case["rows"] if op == "norm" else case["m"]
    s = {"x": _activations(rows, case["k"], g, _DT[case["dtype"]] if op == "norm" else torch.bfloat16)}
    if op in ("norm", "layer"):
        s["weight"] = _normal((case["k"],), g, 0.1) + 1.0
        res = case["res"] if op == "norm" else "bf16"
        if res != "none":
            s["res"] = _normal((rows, case["k"]), g, 2.0, _DT[res])
    if op != "norm":
        s["w"] = _normal((case["o"], case["k"]), g, math.sqrt(2.0 / case["k"]))
    return s


# ---- the operators in plain torch operations ------------------------------------------------------------------------

def _plain_quantize(x):
    """E4M3 codes of whole blocks, the last one filled with zeros, and biased scale exponents, one per block."""
    x = x.float()
    fill = -x.shape[-1] % BLOCK
    if fill:
        x = torch.cat([x, x.new_zeros(x.shape[:-1] + (fill,))], -1)
    y = x.reshape(x.shape[:-1] + (-1, BLOCK))
    e = ((y.abs().amax(-1, keepdim=True).view(torch.int32) + 0x1FFFFF >> 23) - 8).clamp_min(0)
    y = y * ((254 - e) << 23).view(torch.float32)
    return y.to(torch.float8_e4m3fn), e.squeeze(-1).to(torch.uint8)


def _plain_values(code, e):
    """What codes and scale exponents stand for, fp32."""
    scale = torch.maximum(e.int() << 23, torch.full_like(e, 0, dtype=torch.int32) + 0x00400000).view(torch.float32)
    return (code.float() * scale.unsqueeze(-1)).flatten(-2)


def _plain_norm(s):
    """(x + residual, its norm), fp32."""
    h = s["x"].float()
    if "res" in s:
        h = h + s["res"].float()
    return h, h * torch.rsqrt(h.square().mean(-1, keepdim=True) + _EPS) * s["weight"].float()


def _plain_rotate(s):
    case = s["case"]
    p, x = case["pairs"], s["qkv"][:, :, : case["heads"]].float()
    # 64 bits: an angle of a million radians in 32 is off by a sixteenth of one
    freq = _THETA ** (-torch.arange(p, dtype=torch.float64, device=x.device) / p)
    angle = s["positions"].double()[s["axis_of"]].permute(1, 2, 0) * freq
    cos, sin = torch.cos(angle).float()[:, :, None], torch.sin(angle).float()[:, :, None]
    if case["adjacent"]:
        a, b = x[..., 0:2 * p:2], x[..., 1:2 * p:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = x[..., :p], x[..., p:2 * p]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([turned, x[..., 2 * p:]], -1).to(s["qkv"].dtype)


# ---- state --------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    op, dev = case["op"], _device()
    if own:
        from paper_2105_09377_b200 import binding as gl
        ap = gl.AccessPattern
        flags = (gl.GL_EPILOGUE_RELU if case.get("relu") else 0) | (gl.GL_OUT_BF16 if case.get("out") == "bf16" else 0)
    if op == "quantize":
        if own:
            # the program keeps its buffers and its two prepared calls
            q = gl.f8_empty(tuple(s["x"].shape), 1, dev)
            s["result"] = torch.empty_like(s["x"])
            s["calls"] = [gl.prepare_f8_quantize(ap(s["x"], 1), q), gl.prepare_f8_dequantize(q, ap(s["result"], 1))]
        return s
    if op == "rotate":
        if own:
            plan = gl.rotary_plan(case["pairs"], _THETA, _sections(case), adjacent=case["adjacent"])
            part = s["qkv"][:, :, : case["heads"]]                   # queries and keys, read where they are
            s["result"] = torch.empty(part.shape, dtype=part.dtype, device=dev)
            s["calls"] = [gl.prepare_compute_rotate(ap(part, 3), plan, s["positions"], ap(s["result"], 3))]
        else:
            s["axis_of"] = torch.tensor([a for a, n in enumerate(_sections(case)) for _ in range(n)], device=dev)
        return s
    if op != "norm":
        # weights (and, for the product, the left operand) are laid out once
        if own:
            w = gl.gl_f8_quantize(ap(s["w"], 1))
            result = ap(torch.empty((case["m"], case["o"]), dtype=_DT[case["out"]], device=dev), 2)
        else:
            s["w_codes"], s["w_exps"] = _plain_quantize(s["w"])
            if op == "product":
                s["x_codes"], s["x_exps"] = _plain_quantize(s["x"])
                del s["x"]
        del s["w"]
    if own and op == "dense":
        s["result"], s["calls"] = result.tensor, [gl.prepare_dense_f8(ap(s["x"], 1), w, result, flags)]
    elif own and op == "product":
        s["result"], s["calls"] = result.tensor, [gl.prepare_cartesian_dot_f8(gl.gl_f8_quantize(ap(s["x"], 1)), w, result, flags)]
    elif own:
        x, weight, shape = ap(s["x"], 1), ap(s["weight"], 0), tuple(s["x"].shape)
        res = ap(s["res"], 1) if "res" in s else None
        total = ap(torch.empty_like(s["res"]), 1) if "res" in s else None
        eight = op == "layer" or case["out"] == "f8"
        y = gl.f8_empty(shape, 1, dev) if eight else ap(torch.empty(shape, dtype=_DT[case["out"]], device=dev), 1)
        s["calls"] = [gl.prepare_compute_norm_rms(x, weight, y, _EPS, res, total)]
        if op == "layer":
            s["calls"].append(gl.prepare_cartesian_dot_f8(y, w, result, flags))
            s["result"] = [total.tensor, result.tensor]
        else:
            back = ap(torch.empty(shape, dtype=torch.bfloat16, device=dev), 1) if eight else y
            if eight:
                s["calls"].append(gl.prepare_f8_dequantize(y, back))
            s["result"] = ([total.tensor] if total is not None else []) + [back.tensor]
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------

def run(s):
    if own:
        for call in s["calls"]:
            call()
        return s["result"]
    case = s["case"]
    op = case["op"]
    if op == "quantize":
        return _plain_values(*_plain_quantize(s["x"]))[:, : case["k"]].to(s["x"].dtype)
    if op == "rotate":
        return _plain_rotate(s)
    if op == "norm":
        h, y = _plain_norm(s)
        if case["out"] == "f8":
            y = _plain_values(*_plain_quantize(y))[:, : case["k"]].to(torch.bfloat16)
        else:
            y = y.to(_DT[case["out"]])
        return ([h.to(s["res"].dtype)] if "res" in s else []) + [y]
    if op == "product":
        x = _plain_values(s["x_codes"], s["x_exps"])
    elif op == "dense":
        x = _plain_values(*_plain_quantize(s["x"]))
    else:
        h, y = _plain_norm(s)
        x = _plain_values(*_plain_quantize(y))
    y = x @ _plain_values(s["w_codes"], s["w_exps"]).t()
    y = (y.clamp_min(0.0) if case["relu"] else y).to(_DT[case["out"]])
    return [h.to(s["res"].dtype), y] if op == "layer" else y


# ---- what a pass cannot do without ---------------------------------------------------------------------------------

_ES = {"bf16": 2, "f32": 4, "none": 0}


def _held(rows, k):
    return rows * (k + -(-k // BLOCK))


def work(case):
    op = case["op"]
    if op == "quantize":
        return {"bytes": 2 * _ES[case["dtype"]] * case["rows"] * case["k"] + 2 * _held(case["rows"], case["k"]), "flops": 0}
    if op == "norm":
        rows, k = case["rows"], case["k"]
        out = 2 * _held(rows, k) + 2 * rows * k if case["out"] == "f8" else _ES[case["out"]] * rows * k
        return {"bytes": (_ES[case["dtype"]] + 2 * _ES[case["res"]]) * rows * k + 2 * k + out, "flops": 0}
    if op == "rotate":
        n = case["batch"] * case["t"]
        return {"bytes": 2 * _ES[case["dtype"]] * n * case["heads"] * case["d"] + 4 * case["axes"] * n, "flops": 0}
    m, k, o = case["m"], case["k"], case["o"]
    left = {"product": _held(m, k), "dense": 2 * m * k, "layer": 6 * m * k + 2 * k}[op]   # (layer: x, residual and sum)
    return {"bytes": left + _held(o, k) + _ES[case["out"]] * m * o, "flops": 2 * m * k * o}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def _exact_values(x):
    """[..., K] rounded to the format, by nearest multiples of the step of each value's binade."""
    k = x.shape[-1]
    x = torch.nn.functional.pad(x.double(), (0, -k % BLOCK))
    y = x.unflatten(-1, (-1, BLOCK))
    top = torch.frexp(y.abs().amax(-1, keepdim=True))           # mantissa in [0.5, 1): 1.75 there is 0.875 here
    e = top.exponent - 9 + (top.mantissa > 0.875).int()
    e = torch.where(top.mantissa > 0, e, -127).clamp_min(-127).double()
    y = y / torch.exp2(e)
    step = torch.exp2((torch.frexp(y).exponent - 1).clamp_min(-6).double() - 3)
    return (torch.round(y / step) * step * torch.exp2(e)).flatten(-2)[..., :k]


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "quantize":
        return _exact_values(s["x"])
    if op == "rotate":
        p, x = case["pairs"], s["qkv"][:, :, : case["heads"]].double()
        unit = torch.exp(-math.log(_THETA) / p * torch.arange(p, dtype=torch.float64, device=x.device))
        where = torch.repeat_interleave(torch.arange(case["axes"], device=x.device), torch.tensor(_sections(case), device=x.device))
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=x.device), s["positions"].double()[where].movedim(0, -1) * unit)
        head = x[..., : 2 * p].unflatten(-1, (p, 2) if case["adjacent"] else (2, p))
        if not case["adjacent"]:
            head = head.transpose(-1, -2)
        head = torch.view_as_real(torch.view_as_complex(head.contiguous()) * turn[:, :, None])
        if not case["adjacent"]:
            head = head.transpose(-1, -2)
        out = x.clone()
        out[..., : 2 * p] = head.flatten(-2)
        return out
    x = s["x"].double()
    if op in ("norm", "layer"):
        total = x + s["res"].double() if "res" in s else x
        x = total / torch.sqrt(total.pow(2).sum(-1, keepdim=True) / case["k"] + _EPS) * s["weight"].double()
        if op == "norm":
            return ([total] if "res" in s else []) + [_exact_values(x) if case["out"] == "f8" else x]
    y = _exact_values(x) @ _exact_values(s["w"]).t()
    y = torch.relu(y) if case["relu"] else y
    return [total, y] if op == "layer" else y
