"""Cases of the 4-bit operators: blocks of 32 values with one power-of-two scale (MX4), the product of such operands,
and attention over a cache of keys and values held that way.

Number format (one block = 32 consecutive values of an item): with a = max |v|, the scale is 2^(floor(log2 a) - 2), never
below 2^-127; each value divided by the scale is rounded to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (ties to the even
mantissa, larger values to 6) and keeps its sign.

`run` computes one pass either in plain torch operations, in 32 bits (`own` false), or through the library's calls.
"""
import math

import torch

own = False

BLOCK = 32
_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- cases --------------------------------------------------------------------------------------------------------

def listed():
    return [
        # rows that end inside a block, fp32 results of another layer
        {"name": "quantize_odd", "op": "quantize", "rows": 777, "k": 1111, "dtype": "f32"},
        # a large layer's activations (or its weights, once)
        {"name": "quantize_large", "op": "quantize", "rows": 16384, "k": 8192, "dtype": "bf16"},
        # a dense layer at one token: the weights are read once, nothing is reused
        {"name": "dense_token", "op": "dense", "m": 1, "k": 8192, "o": 8192, "relu": False, "out": "bf16"},
        # the 3136 -> 1000 layer that ends the framework's stem chain, at its batch of 32, fp32 logits
        {"name": "dense_chain", "op": "dense", "m": 32, "k": 3136, "o": 1000, "relu": False, "out": "f32"},
        # both operands already in 4 bits, nothing a multiple of anything
        {"name": "product_odd", "op": "product", "m": 301, "k": 1111, "o": 777, "relu": True, "out": "bf16"},
        # the framework's headline product with both operands held in 4 bits
        {"name": "product_4096", "op": "product", "m": 4096, "k": 4096, "o": 4096, "relu": True, "out": "f32"},
        # a prompt's worth of tokens through a large layer
        {"name": "dense_large", "op": "dense", "m": 16384, "k": 8192, "o": 8192, "relu": False, "out": "bf16"},
        # one step of a batch in flight: a token per sequence is stored and read back (what a check of the cache does)
        {"name": "append_token", "op": "append", "batch": 64, "t": 1, "hkv": 8, "d": 128, "page": 64, "lo": 17, "hi": 4096},
        # prompts of different lengths enter the cache (left-padded to the longest)
        {"name": "append_prompt", "op": "append", "batch": 4, "t": 2047, "hkv": 8, "d": 128, "page": 16, "lo": 700, "hi": 2047},
        # one short conversation, a query head per key head
        {"name": "attend_short", "op": "attend", "batch": 1, "t": 1, "hq": 8, "hkv": 8, "d": 64, "page": 16, "lo": 33, "hi": 33, "out": "f32"},
        # a batch in flight, four query heads per key head, from 17 tokens to 16384
        {"name": "attend_batch", "op": "attend", "batch": 16, "t": 1, "hq": 32, "hkv": 8, "d": 128, "page": 64, "lo": 17, "hi": 16384, "out": "bf16"},
        # 512 tokens of two prompts that are read in pieces, behind what is already in the cache
        {"name": "attend_prompt", "op": "attend", "batch": 2, "t": 512, "hq": 32, "hkv": 8, "d": 128, "page": 64, "lo": 5001, "hi": 8192, "out": "bf16"},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["quantize", "dense", "dense", "product", "append", "attend", "attend", "attend"])
    if op == "quantize":
        rows = _log(rng, 1, 16384)
        return {"op": op, "rows": rows, "k": _log(rng, 1, min(16384, 16384 * 8192 // rows)), "dtype": rng.choice(["bf16", "f32"])}
    if op in ("dense", "product"):
        return {"op": op, "m": _log(rng, 1, 16384), "k": _log(rng, 17, 8192), "o": _log(rng, 9, 8192),
                "relu": rng.random() < 0.5, "out": rng.choice(["bf16", "f32"])}
    hkv, d, page = rng.choice([1, 2, 4, 8]), rng.choice([64, 128, 256]), rng.choice([16, 32, 64, 128])
    if op == "append":
        t = _log(rng, 1, 2047)
        batch = _log(rng, 1, max(1, min(256, 8192 // t)))
        hi = _log(rng, t, 4096)
        return {"op": op, "batch": batch, "t": t, "hkv": hkv, "d": d, "page": page, "lo": rng.randint(max(0, t // 2), hi), "hi": hi}
    batch = _log(rng, 1, 64)
    hi = _log(rng, 1, min(131072, 64 * 4096 * 8 * 128 // (batch * hkv * d)))
    group = rng.choice([1, 2, 4, 5, 8, 16])
    most = max(1, min(512, 2 ** 28 // (batch * group * hkv * hi)))
    t = 1 if rng.random() < 0.6 else _log(rng, 1, most)
    return {"op": op, "batch": batch, "t": t, "hq": hkv * group, "hkv": hkv, "d": d, "page": page,
            "lo": rng.randint(0, hi), "hi": hi, "out": rng.choice(["bf16", "f32"])}


def _lengths(case):
    """Tokens in the cache per sequence, the new ones included: from `lo` to `hi`, evenly spread."""
    b = case["batch"]
    return [case["hi"] - (case["hi"] - case["lo"]) * i // max(1, b - 1) for i in range(b)]


def _visible(case):
    """Keys that the rows of one sequence see together (row i of t sees the keys up to its own position)."""
    return _lengths(case)


# ---- inputs: what a program has in hand ---------------------------------------------------------------------------

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
    g = torch.Generator(device=_device()).manual_seed(1000003 * int(seed) + 17)
    op = case["op"]
    if op == "quantize":
        return {"x": _activations(case["rows"], case["k"], g, _DT[case["dtype"]])}
    if op in ("dense", "product"):
        return {"x": _activations(case["m"], case["k"], g, torch.bfloat16),
                "w": _normal((case["o"], case["k"]), g, math.sqrt(2.0 / case["k"]))}
    lens = _lengths(case)
    page, hkv, d, b = case["page"], case["hkv"], case["d"], case["batch"]
    width = max(1, -(-max(lens) // page))
    table = torch.randperm(b * width, generator=g, device=g.device).to(torch.int32).reshape(b, width)
    r = {"table": table, "lengths": torch.tensor(lens, dtype=torch.int32, device=g.device)}
    n = case["t"] if op == "append" else max(1, max(lens))
    channel = torch.exp(0.7 * torch.randn((hkv, d), generator=g, device=g.device))   # keys: channels of unequal size
    r["k"] = (torch.randn((b, n, hkv, d), generator=g, device=g.device) * channel).to(torch.bfloat16)
    r["v"] = _normal((b, n, hkv, d), g)
    if op == "attend":
        r["q"] = _normal((b, case["t"], case["hq"], d), g, 1.5)
    return r


# ---- the format in plain torch operations -------------------------------------------------------------------------

def _blocks(x):
    """[..., K] -> fp32 [..., blocks, 32], the last block filled with zeros."""
    x = x.float()
    fill = -x.shape[-1] % BLOCK
    if fill:
        x = torch.cat([x, x.new_zeros(x.shape[:-1] + (fill,))], -1)
    return x.reshape(x.shape[:-1] + (-1, BLOCK))


def _plain_quantize(x):
    """Codes (sign, 3 bits of magnitude) one to a byte, and biased scale exponents, one per block."""
    y = _blocks(x)
    top = y.abs().amax(-1, keepdim=True).view(torch.int32) >> 23
    e = (top - 2).clamp_min(0)
    y = y * ((254 - e) << 23).view(torch.float32)
    a = y.abs()
    code = (a > 0.25).to(torch.uint8)
    code += a >= 0.75
    code += a > 1.25
    code += a >= 1.75
    code += a > 2.5
    code += a >= 3.5
    code += a > 5.0
    code |= torch.signbit(y).to(torch.uint8) << 3
    return code.flatten(-2), e.squeeze(-1).to(torch.uint8)


def _plain_values(code, e):
    """What codes and scale exponents stand for, fp32."""
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=code.device)
    mag = table[(code & 7).int()]
    val = torch.where((code & 8) != 0, -mag, mag).reshape(e.shape + (BLOCK,))
    scale = torch.maximum(e.int() << 23, torch.full_like(e, 0, dtype=torch.int32) + 0x00400000).view(torch.float32)
    return (val * scale.unsqueeze(-1)).flatten(-2)


def _two_to_a_byte(code):
    return code[..., 0::2] | (code[..., 1::2] << 4)


def _one_to_a_byte(packed):
    return torch.stack([packed & 15, packed >> 4], -1).flatten(-2)


def _positions(lengths, t):
    """Cache position of each of the last t tokens of each sequence; negative: left padding, not in the cache."""
    return lengths[:, None].long() - t + torch.arange(t, device=lengths.device)


def _slots(s, pos):
    """(page, place in it) of cache positions [batch, n]."""
    page = s["case"]["page"]
    return s["table"].gather(1, (pos // page).clamp(0, s["table"].shape[1] - 1)).long(), pos % page


def _plain_append(s, k, v, pos):
    keep = pos >= 0
    pg, at = (i[keep] for i in _slots(s, pos.clamp_min(0)))
    for name, x in (("k", k), ("v", v)):
        code, e = _plain_quantize(x[keep])
        s[name + "_codes"][pg, at] = _two_to_a_byte(code)
        s[name + "_exps"][pg, at] = e


def _plain_gather(s, name, pos):
    pg, at = _slots(s, pos)
    return _plain_values(_one_to_a_byte(s[name + "_codes"][pg, at]), s[name + "_exps"][pg, at])


# ---- state --------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    op, dev = case["op"], _device()
    if own:
        from paper_2105_09377_b200 import binding as gl
        flags = (gl.GL_EPILOGUE_RELU if case.get("relu") else 0) | (gl.GL_OUT_BF16 if case.get("out") == "bf16" else 0)
    if op == "quantize":
        if own:
            # the program keeps its buffers and its two prepared calls
            q = gl.mx4_empty(tuple(s["x"].shape), 1, dev)
            s["result"] = gl.AccessPattern(torch.empty_like(s["x"]), 1)
            s["calls"] = [gl.prepare_mx4_quantize(gl.AccessPattern(s["x"], 1), q), gl.prepare_mx4_dequantize(q, s["result"])]
    elif op in ("dense", "product"):
        # weights (and, for the product, the left operand) are laid out once
        if own:
            w = gl.gl_mx4_quantize(gl.AccessPattern(s["w"], 1))
            s["result"] = gl.AccessPattern(torch.empty((case["m"], case["o"]), dtype=_DT[case["out"]], device=dev), 2)
            x = gl.AccessPattern(s["x"], 1)
            if op == "dense":
                s["calls"] = [gl.prepare_dense_mx4(x, w, s["result"], flags)]
            else:
                s["calls"] = [gl.prepare_cartesian_dot_mx4(gl.gl_mx4_quantize(x), w, s["result"], flags)]
        else:
            s["w_codes"], s["w_exps"] = _plain_quantize(s["w"])
            s["w_codes"] = _two_to_a_byte(s["w_codes"])
            if op == "product":
                s["x_codes"], s["x_exps"] = _plain_quantize(s["x"])
                s["x_codes"] = _two_to_a_byte(s["x_codes"])
                del s["x"]
        del s["w"]
    else:
        pages, page, hkv, d = s["table"].numel(), case["page"], case["hkv"], case["d"]
        n = s["k"].shape[1]
        if own:
            cache = gl.cache4_empty(pages, hkv, page, d, dev)
            append = gl.prepare_cache4_append(cache, s["k"], s["v"], s["table"], s["lengths"])
            if op == "append":
                s["result"] = [torch.empty_like(s["k"]), torch.empty_like(s["v"])]
                s["calls"] = [append, gl.prepare_cache4_read(cache, s["result"][0], s["result"][1], s["table"], s["lengths"])]
            else:
                append()
                s["result"] = gl.AccessPattern(torch.empty(s["q"].shape, dtype=_DT[case["out"]], device=dev), 3)
                s["calls"] = [gl.prepare_attend_cache4(gl.AccessPattern(s["q"], 3), cache, s["table"], s["lengths"], s["result"],
                                                       1.0 / math.sqrt(d), flags)]
        else:
            for name in "kv":
                s[name + "_codes"] = torch.zeros((pages, page, hkv, d // 2), dtype=torch.uint8, device=dev)
                s[name + "_exps"] = torch.zeros((pages, page, hkv, d // BLOCK), dtype=torch.uint8, device=dev)
            if op == "attend":
                _plain_append(s, s["k"], s["v"], _positions(s["lengths"], n))
        if op == "attend":
            del s["k"], s["v"]
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------

def run(s):
    if own:
        for call in s["calls"]:
            call()
        r = s["result"]
        return r if isinstance(r, list) else r.tensor
    case = s["case"]
    op = case["op"]
    if op == "quantize":
        return _plain_values(*_plain_quantize(s["x"]))[:, : case["k"]].to(s["x"].dtype)
    if op in ("dense", "product"):
        w = _plain_values(_one_to_a_byte(s["w_codes"]), s["w_exps"])
        x = _plain_values(*_plain_quantize(s["x"])) if op == "dense" else _plain_values(_one_to_a_byte(s["x_codes"]), s["x_exps"])
        y = x @ w.t()
        return (y.clamp_min(0.0) if case["relu"] else y).to(_DT[case["out"]])
    t = case["t"]
    pos = _positions(s["lengths"], t)
    if op == "append":
        _plain_append(s, s["k"], s["v"], pos)
        there = (pos >= 0)[:, :, None, None]
        return [torch.where(there, _plain_gather(s, name, pos.clamp_min(0)), 0.0).to(torch.bfloat16) for name in "kv"]
    n = max(1, case["hi"])
    every = torch.arange(n, device=pos.device).expand(case["batch"], n)
    k, v = (_plain_gather(s, name, every).transpose(1, 2) for name in "kv")             # [b, hkv, n, d]
    b, hkv, d = case["batch"], case["hkv"], case["d"]
    group = case["hq"] // hkv
    q = s["q"].float().reshape(b, t, hkv, group, d).permute(0, 2, 3, 1, 4).reshape(b, hkv, group * t, d)
    seen = (every[:, None, :] <= pos[:, :, None])[:, None, None].expand(b, 1, group, t, n).reshape(b, 1, group * t, n)
    score = torch.where(seen, q @ k.transpose(2, 3) * (1.0 / math.sqrt(d)), float("-inf"))
    top = score.amax(-1, keepdim=True).clamp_min(torch.finfo(torch.float32).min)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    y = (p @ torch.where(seen.any(2)[..., None], v, 0.0)) / torch.where(total > 0, total, 1.0)
    return y.reshape(b, hkv, group, t, d).permute(0, 3, 1, 2, 4).reshape(b, t, case["hq"], d).to(_DT[case["out"]])


# ---- what a pass cannot do without ---------------------------------------------------------------------------------

def _held(values, blocks):
    return values / 2 + blocks


def work(case):
    op = case["op"]
    es = {"bf16": 2, "f32": 4}
    if op == "quantize":
        n, nb = case["rows"] * case["k"], case["rows"] * -(-case["k"] // BLOCK)
        return {"bytes": 2 * es[case["dtype"]] * n + 2 * _held(n, nb), "flops": 0}
    if op in ("dense", "product"):
        m, k, o = case["m"], case["k"], case["o"]
        nb = -(-k // BLOCK)
        left = 2 * m * k if op == "dense" else _held(m * k, m * nb)
        return {"bytes": left + _held(o * k, o * nb) + es[case["out"]] * m * o, "flops": 2 * m * k * o}
    hkv, d = case["hkv"], case["d"]
    token = 2 * hkv * _held(d, d // BLOCK)      # keys and values of one token
    lens = _lengths(case)
    if op == "append":
        stored = sum(min(n, case["t"]) for n in lens)
        # read k and v, write the cache, read it back, write every token of the results
        return {"bytes": stored * (2 * hkv * d * 2 + 2 * token) + case["batch"] * case["t"] * 2 * hkv * d * 2, "flops": 0}
    pairs = sum(max(0, n - i) for n in lens for i in range(case["t"]))
    q = case["batch"] * case["t"] * case["hq"] * d
    return {"bytes": sum(_visible(case)) * token + q * (2 + es[case["out"]]), "flops": 4 * pairs * case["hq"] * d}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def _exact_values(x):
    """[..., K] rounded to the format, by nearest multiples of the step of each value's binade."""
    k = x.shape[-1]
    x = torch.nn.functional.pad(x.double(), (0, -k % BLOCK))
    y = x.unflatten(-1, (-1, BLOCK))
    top = torch.frexp(y.abs().amax(-1, keepdim=True))
    e = torch.where(top.mantissa > 0, top.exponent - 1 - 2, -127).clamp_min(-127).double()
    y = y / torch.exp2(e)
    step = torch.exp2((torch.frexp(y).exponent - 1).clamp_min(0).double() - 1)   # half a unit below 1, as below 2
    y = torch.minimum(torch.round(y.abs() / step) * step, torch.full_like(y, 6.0)) * torch.sign(y)
    return (y * torch.exp2(e)).flatten(-2)[..., :k]


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "quantize":
        return _exact_values(s["x"])
    if op in ("dense", "product"):
        y = _exact_values(s["x"]) @ _exact_values(s["w"]).t()
        return torch.relu(y) if case["relu"] else y
    lens, t = _lengths(case), case["t"]
    if op == "append":
        out = []
        for name in "kv":
            y = _exact_values(s[name])
            for i, n in enumerate(lens):
                y[i, : max(0, t - n)] = 0
            out.append(y)
        return out
    group, d, wide = case["hq"] // case["hkv"], case["d"], s["k"].shape[1]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    for i, n in enumerate(lens):
        if n == 0:
            continue
        k, v = _exact_values(s["k"][i, wide - n:]), _exact_values(s["v"][i, wide - n:])
        own_place = n - t + torch.arange(t, device=k.device)
        rows = own_place >= 0
        hidden = torch.arange(n, device=k.device)[None, :] > own_place[rows][:, None]
        for h in range(case["hq"]):
            a = s["q"][i, rows, h].double() @ k[:, h // group].t() / math.sqrt(d)
            out[i, rows, h] = torch.softmax(a.masked_fill(hidden, float("-inf")), -1) @ v[:, h // group]
    return out
