"""The operators of linear and expert layers in 4-bit floating point whose speed is measured.

A number is a 4-bit value (1-2-1 bits: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) times the scale of its block along the row, in
one of two formats:

* ``mx``: blocks of 32, a power of two in 8 bits (E8M0) for each;
* ``nv``: blocks of 16, an E4M3 scale for each, and one fp32 factor for the whole tensor.

Four kinds of case:

* ``quantise``: a matrix to 4 bits and back to the values that they stand for (two calls);
* ``dequantise``: stored 4-bit values and scales to 16 or 32 bits;
* ``matmul``: the product of two such matrices, alone or one for each group of consecutive rows (an expert's tokens);
* ``experts``: a gated feed-forward layer of routed experts with 4-bit weights, from the tokens and their routes to its output.

The plain form is written with elementary torch operations in 32 bits (in 64 where a value next to a border decides a 4-bit
result), the other side is the package's own calls.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "f16": 2, "bf16": 2}
_BLOCK = {"mx": 32, "nv": 16}


# ---- cases -----------------------------------------------------------------------------------------------------------

def listed():
    return [
        # The activations of one token on their way into a linear layer: the smallest call.
        dict(name="quantise_1x4096", kind="quantise", rows=1, cols=4096, format="nv", factor=True, x="bf16"),
        # The activations of a long prompt or a large batch.
        dict(name="quantise_16384x8192", kind="quantise", rows=16384, cols=8192, format="nv", factor=True, x="bf16"),
        # A weight matrix when a model is loaded; its last block is not full and its rows have an odd number of values.
        dict(name="quantise_8203x5137", kind="quantise", rows=8203, cols=5137, format="mx", factor=False, x="f32"),
        # A small matrix with ragged rows, looked at in 16 bits.
        dict(name="dequantise_37x4111", kind="dequantise", rows=37, cols=4111, format="mx", factor=False, x="f16"),
        # A stored weight matrix for a layer that computes in 16 bits.
        dict(name="dequantise_8192x8192", kind="dequantise", rows=8192, cols=8192, format="nv", factor=True, x="bf16"),
        # One token through a linear layer: every weight is read for one row.
        dict(name="matmul_1x8192x8192", kind="matmul", rows=1, n=8192, k=8192, groups=1, format="nv", y="bf16"),
        # A small batch of sequences decoded together, odd sizes.
        dict(name="matmul_37x5136x4128", kind="matmul", rows=37, n=5136, k=4128, groups=1, format="mx", y="f16"),
        # A long prompt through a large layer: bound by arithmetic.
        dict(name="matmul_8192x8192x8192", kind="matmul", rows=8192, n=8192, k=8192, groups=1, format="nv", y="bf16"),
        # Rows sorted by expert, each expert with a weight matrix of its own; ragged groups, some empty.
        dict(name="matmul_8192x2048x4096_g32", kind="matmul", rows=8192, n=2048, k=4096, groups=32, format="mx", y="bf16"),
        # One token through an expert layer: a few experts' weights are read for one row each.
        dict(name="experts_1_of_64", kind="experts", tokens=1, experts=64, topk=4, hidden=2048, inter=1024, format="mx", x="bf16"),
        # A small batch decoded together through the same layer.
        dict(name="experts_16_of_64", kind="experts", tokens=16, experts=64, topk=4, hidden=2048, inter=1024, format="nv", x="bf16"),
        # A long prompt through it: bound by arithmetic.
        dict(name="experts_8192_of_64", kind="experts", tokens=8192, experts=64, topk=4, hidden=2048, inter=1024, format="nv", x="bf16"),
    ]


def _log(rng, lo, hi):
    """An integer between lo and hi, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["quantise", "quantise", "dequantise", "matmul", "matmul", "matmul", "experts", "experts", "experts"])
    fmt = rng.choice(["mx", "nv"])
    if kind in ("quantise", "dequantise"):
        cols = _log(rng, 100, 8192)
        if rng.random() < 0.5:
            cols = (cols + 31) // 32 * 32
        x = rng.choice(["bf16", "bf16", "f16", "f32"])
        return dict(kind=kind, rows=_log(rng, 1, min(16384, 260e6 / cols / _SIZE[x])), cols=cols, format=fmt,
                    factor=fmt == "nv" and rng.random() < 0.7, x=x)
    if kind == "matmul":
        groups = rng.choice([1, 1, 1, rng.randint(2, 64)])
        n, k = _log(rng, 64, 8192), 32 * _log(rng, 4, 256)
        if rng.random() < 0.5:
            n = (n + 63) // 64 * 64
        if groups > 1:
            n, k = min(n, 4096), min(k, 4096)
            groups = min(groups, max(2, (1 << 28) // (n * k)))
        return dict(kind=kind, rows=_log(rng, 1, 8192), n=n, k=k, groups=groups, format=fmt, y=rng.choice(["bf16", "bf16", "f16", "f32"]))
    return dict(kind=kind, tokens=_log(rng, 1, 8192), experts=rng.choice([8, 16, 24, 32, 64]), topk=rng.randint(1, 4), hidden=32 * _log(rng, 8, 64),
                inter=32 * _log(rng, 4, 32), format=fmt, x=rng.choice(["bf16", "bf16", "f16"]))


def _blocks(n, fmt):
    return -(-n // _BLOCK[fmt])


def _active(tokens, experts, topk):
    """Expected number of experts that get a token, each token taking `topk` different ones."""
    return experts * (1.0 - (1.0 - topk / experts) ** tokens)


def work(case):
    c, fmt = case, case["format"]
    if c["kind"] in ("quantise", "dequantise"):
        packed = c["rows"] * ((c["cols"] + 1) // 2 + _blocks(c["cols"], fmt))
        wide = c["rows"] * c["cols"] * _SIZE[c["x"]]
        both = 2 if c["kind"] == "quantise" else 1  # there and back: x is read, the packed form written and read, y written
        return {"bytes": both * (packed + wide), "flops": both * 2 * c["rows"] * c["cols"]}
    if c["kind"] == "matmul":
        rows = c["rows"] - (c["rows"] // 16 if c["groups"] > 1 else 0)  # the rest belongs to no group
        weights = 1 if c["groups"] == 1 else max(1, min(c["groups"] - 1, rows))
        row = c["k"] // 2 + _blocks(c["k"], fmt)
        return {"bytes": rows * (row + c["n"] * _SIZE[c["y"]]) + weights * c["n"] * row, "flops": 2 * rows * c["n"] * c["k"]}
    matrix = c["hidden"] * c["inter"]
    return {"bytes": 3 * matrix * (0.5 + 1 / _BLOCK[fmt]) * _active(c["tokens"], c["experts"], c["topk"]) +
            c["tokens"] * (2 * c["hidden"] * _SIZE[c["x"]] + 8 * c["topk"]), "flops": 6 * matrix * c["tokens"] * c["topk"]}


# ---- plain forms -----------------------------------------------------------------------------------------------------

def _round4(v):
    """The nearest 4-bit value (ties to even): steps of 0.5 below 2, of 1 below 4, of 2 up to 6."""
    a = v.abs()
    step = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0)).to(v.dtype)
    return torch.copysign((torch.round(a / step) * step).clamp_max(6.0), v)


def _quantise(x, fmt, factor, precise=True):
    """(4-bit values in x's shape, scales in 8 bits) of a matrix, every row in blocks.  The borders between neighbouring values are met in 64
    bits, unless nobody looks where next to them a value goes (weights made up from random numbers)."""
    rows, cols = x.shape
    b = _BLOCK[fmt]
    p = x.to(torch.float64 if precise else torch.float32)
    p = torch.nn.functional.pad(p, (0, -cols % b)).reshape(rows, -1, b)
    amax = p.abs().amax(-1)
    g = (factor if factor is not None else torch.ones(1, device=x.device)).to(p.dtype)  # (a tensor: by a number torch divides as by its reciprocal)
    if fmt == "mx":  # the least power of two that keeps the block within 6
        m, e = torch.frexp(amax)  # amax = m 2^e, m in [0.5, 1)
        e = torch.where(amax > 0, torch.where(m <= 0.75, e - 3, e - 2), -127).clamp(-127, 127)
        scale = (e + 127).to(torch.uint8)
        step = torch.ldexp(torch.ones_like(amax), e)
    else:
        scale = (amax / (6.0 * g)).clamp_max(448.0)
        # (to E4M3 by hand, as a conversion would round to 32 bits first)
        _, e = torch.frexp(scale)
        grain = torch.ldexp(torch.ones_like(scale), (e - 1).clamp_min(-6) - 3)
        scale = (torch.round(scale / grain) * grain).clamp_max(448.0)
        step = scale * g
        scale = scale.float().to(torch.float8_e4m3fn).view(torch.uint8)
    v = torch.where(step[..., None] > 0, p / step[..., None], 0.0)
    return _round4(v).reshape(rows, -1)[:, :cols], scale


_SCALES = {"mx": torch.float8_e8m0fnu, "nv": torch.float8_e4m3fn}


def _numbers(scale, fmt):
    """Scales from their 8 bits, in 32."""
    if fmt == "nv":
        return scale.contiguous().view(torch.float8_e4m3fn).float()
    return torch.ldexp(torch.ones_like(scale, dtype=torch.float32), scale.int() - 127)


def _pack(v):
    """4-bit values (0.5 steps of sign and magnitude) two to a byte, the even column in the low half; a row of odd length ends with a zero."""
    a = v.abs()
    code = torch.where(a < 2.0, 2 * a, torch.where(a < 4.0, a + 2, a / 2 + 4)).to(torch.uint8)
    code |= torch.signbit(v).to(torch.uint8) << 3
    code = torch.nn.functional.pad(code, (0, v.shape[-1] % 2))
    return code[..., 0::2] | (code[..., 1::2] << 4)


_VALUES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]


def _unpack(q, cols):
    """The 4-bit values of packed bytes, in 32 bits."""
    table = torch.tensor([[_VALUES[i & 15], _VALUES[i >> 4]] for i in range(256)], device=q.device)
    return table[q.int()].reshape(*q.shape[:-1], -1)[..., :cols]


def _values(q, scale, fmt, cols):
    """The numbers that 4-bit values and their scales stand for, without the tensor's factor, in 32 bits."""
    s = _numbers(scale, fmt).repeat_interleave(_BLOCK[fmt], -1)[..., :cols]
    return _unpack(q, cols) * s


def _plain_matmul(s, case):
    a, b = _values(s["a"], s["a_scale"], case["format"], case["k"]), _values(s["b"], s["b_scale"], case["format"], case["k"])
    if case["groups"] == 1:
        y = torch.matmul(a, b.t())
        return (y if s["alpha"] is None else y * s["alpha"]).to(s["y"].dtype)
    first, count = s["offsets"][:-1].long(), (s["offsets"][1:] - s["offsets"][:-1]).long()
    at = torch.arange(s["most"], device=a.device)
    index = (first[:, None] + at).clamp_max(a.shape[0] - 1)
    y = torch.matmul(a[index], b.transpose(-1, -2))
    if s["alpha"] is not None:
        y = y * s["alpha"][:, None, None]
    out = torch.zeros(a.shape[0] + 1, case["n"], device=a.device)  # (the last row takes what no group has)
    out[torch.where(at < count[:, None], index, a.shape[0])] = y
    return out[:-1].to(s["y"].dtype)


def _there_and_back(x, fmt, factor):
    """What the 4-bit form of a matrix stands for, in 32 bits."""
    v, scale = _quantise(x, fmt, factor)
    y = v.float() * _numbers(scale, fmt).repeat_interleave(_BLOCK[fmt], -1)[..., :x.shape[1]]
    return y if factor is None else y * factor


def _gated(h):
    gate, up = h.chunk(2, -1)
    return gate / (1.0 + torch.exp(-gate)) * up


def _plain_experts(s, case):
    T, K, E, H, I, fmt = case["tokens"], case["topk"], case["experts"], case["hidden"], case["inter"], case["format"]
    x = _there_and_back(s["x"], fmt, s["x_factor"])
    ids = s["ids"].long()
    f1, f2 = (s[n] if s[n] is not None else torch.ones(E, device=x.device) for n in ("w1_factor", "w2_factor"))
    if T * K <= E:  # few rows: each with its own expert's matrices
        e = ids.reshape(-1)
        w1 = _values(s["w1"][e], s["w1_scale"][e], fmt, H).reshape(T * K, 2 * I, H)
        w2 = _values(s["w2"][e], s["w2_scale"][e], fmt, I)
        h = _gated(torch.matmul(w1, x.repeat_interleave(K, 0)[:, :, None]).squeeze(-1) * f1[e][:, None])
        h = _there_and_back(h, fmt, s["h_factor"])
        y = (torch.matmul(w2, h[:, :, None]).squeeze(-1) * f2[e][:, None]).reshape(T, K, H)
    else:  # all experts at once, each expert's rows padded to the longest
        w1 = _values(s["w1"], s["w1_scale"], fmt, H).reshape(E, 2 * I, H)
        w2 = _values(s["w2"], s["w2_scale"], fmt, I)
        chosen = torch.zeros(T, E, dtype=torch.long, device=x.device).scatter(1, ids, 1)
        place = (chosen.cumsum(0) - chosen).gather(1, ids)  # how many earlier tokens took the same expert
        rows = torch.zeros(E, s["most"], H, device=x.device)
        rows[ids, place] = x[:, None, :].expand(T, K, H)
        h = _gated(torch.matmul(rows, w1.transpose(1, 2)) * f1[:, None, None])
        h = _there_and_back(h.reshape(-1, I), fmt, s["h_factor"]).reshape(E, -1, I)
        y = (torch.matmul(h, w2.transpose(1, 2)) * f2[:, None, None])[ids, place]
    return (y * s["weights"][:, :, None]).sum(1).to(s["y"].dtype)


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _activations(g, *shape):
    """Normal values, one column in about five hundred twenty times larger, as hidden states have them."""
    big = torch.rand(shape[-1], generator=g, device="cuda") < 0.002
    return torch.randn(*shape, generator=g, device="cuda") * torch.where(big, 20.0, 1.0)


def _weights(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda") / math.sqrt(shape[-1])


def _factor(x, fmt):
    """A tensor's factor, with which the largest block gets the largest scale; none where the scales are powers of two."""
    return (x.abs().amax().float() / (6.0 * 448.0)).reshape(1) if fmt == "nv" else None


def _scale_rows(shape, fmt):
    """Room for the scales of rows: each row starts on a multiple of 16 bytes."""
    n = _blocks(shape[-1], fmt)
    return torch.zeros(*shape[:-1], -(-n // 16) * 16, dtype=torch.uint8, device="cuda")[..., :n]


def _stored(x, fmt, factor):
    """(packed values, scales) of a matrix as a program keeps them."""
    v, scale = _quantise(x, fmt, factor, precise=False)
    room = _scale_rows(x.shape, fmt)
    room.copy_(scale)
    return _pack(v), room


def _stored_stack(g, fmt, count, rows, cols):
    """Weights of `count` matrices: (packed values, scales, factors), one matrix after another, so that their 32-bit form is never there whole."""
    q = torch.zeros(count, rows, cols // 2, dtype=torch.uint8, device="cuda")
    scale = _scale_rows((count, rows, cols), fmt)
    factors = torch.ones(count, device="cuda")
    for i in range(count):
        w = _weights(g, rows, cols)
        f = _factor(w, fmt)
        if f is not None:
            factors[i] = f[0]
        q[i], scale[i] = _stored(w, fmt, f)
    return q, scale, factors if fmt == "nv" else None


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s, fmt = {"case": dict(case)}, case["format"]
    if case["kind"] in ("quantise", "dequantise"):
        rows, cols = case["rows"], case["cols"]
        x = _activations(g, rows, cols).to(_TYPES[case["x"]])
        s["factor"] = _factor(x, fmt) if case["factor"] else None
        if case["kind"] == "quantise":
            s["x"] = x
            s["q"] = torch.zeros(rows, (cols + 1) // 2, dtype=torch.uint8, device="cuda")
            s["scale"] = _scale_rows((rows, cols), fmt)
        else:
            s["q"], s["scale"] = _stored(x, fmt, s["factor"])
        s["y"] = torch.zeros(rows, cols, dtype=_TYPES[case["x"]], device="cuda")
    elif case["kind"] == "matmul":
        rows, n, k, groups = case["rows"], case["n"], case["k"], case["groups"]
        x = _activations(g, rows, k)
        fa = _factor(x, fmt)
        s["a"], s["a_scale"] = _stored(x, fmt, fa)
        s["b"], s["b_scale"], fb = _stored_stack(g, fmt, groups, n, k)
        if groups == 1:
            s["b"], s["b_scale"] = s["b"][0], s["b_scale"][0]
        s["alpha"] = fa * fb if fmt == "nv" else None
        s["y"] = torch.zeros(rows, n, dtype=_TYPES[case["y"]], device="cuda")
        s["offsets"], s["most"] = None, 0
        if groups > 1:  # uneven groups, one of them empty, and a few rows behind the last one
            share = torch.exp(0.7 * torch.randn(groups, generator=g, device="cuda"))
            share[torch.randint(groups, (1,), generator=g, device="cuda")] = 0.0
            of = torch.multinomial(share, rows - rows // 16, replacement=True, generator=g)
            count = torch.bincount(of, minlength=groups)
            s["offsets"] = torch.nn.functional.pad(count.cumsum(0), (1, 0)).int()
            s["most"] = int(count.max())
    else:
        T, K, E, H, I = case["tokens"], case["topk"], case["experts"], case["hidden"], case["inter"]
        s["x"] = _activations(g, T, H).to(_TYPES[case["x"]])
        w1, w1_scale, s["w1_factor"] = _stored_stack(g, fmt, E, 2 * I, H)  # gate, then up
        s["w1"], s["w1_scale"] = w1.view(E, 2, I, H // 2), w1_scale.unflatten(1, (2, I))
        s["w2"], s["w2_scale"], s["w2_factor"] = _stored_stack(g, fmt, E, H, I)
        # (factors of the activations as a calibration on other inputs leaves them)
        s["x_factor"], s["h_factor"] = (torch.full((1,), v / (6.0 * 448.0), device="cuda") if fmt == "nv" else None for v in (90.0, 20.0))
        score = torch.rand(T, E, generator=g, device="cuda") + 0.2 * torch.rand(E, generator=g, device="cuda")
        top = score.topk(K, -1)
        s["ids"], s["weights"] = top.indices.int(), top.values / top.values.sum(-1, keepdim=True)
        s["y"] = torch.zeros(T, H, dtype=_TYPES[case["x"]], device="cuda")
        s["most"] = int(torch.bincount(s["ids"].reshape(-1), minlength=E).max())
    return s


# ---- one pass --------------------------------------------------------------------------------------------------------

def run(state):
    s, case = state, state["case"]
    fmt, kind = case["format"], case["kind"]
    if own:
        import paper_2104_04731_b200 as b2c

        typed = lambda scale: scale.view(_SCALES[fmt])  # noqa: E731
        if kind == "quantise":
            b2c.fp4_quantize(s["x"], s["q"], typed(s["scale"]), global_scale=s["factor"])
        if kind in ("quantise", "dequantise"):
            b2c.fp4_dequantize(s["q"], typed(s["scale"]), s["y"], global_scale=s["factor"])
            return {"y": s["y"], "scale": typed(s["scale"])} if kind == "quantise" else s["y"]
        if kind == "matmul":
            b2c.fp4_matmul(s["a"], typed(s["a_scale"]), s["b"], typed(s["b_scale"]), s["y"], alpha=s["alpha"], offsets=s["offsets"])
            return s["y"]
        if "workspace" not in s:
            n = b2c.fp4_experts_workspace_bytes(case["hidden"], case["inter"], case["experts"], case["topk"], case["tokens"],
                                                b2c.MXFP4 if fmt == "mx" else b2c.NVFP4)
            s["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
        b2c.fp4_experts(s["x"], s["ids"], s["weights"], s["w1"], typed(s["w1_scale"]), s["w2"], typed(s["w2_scale"]), s["y"], s["workspace"],
                        x_global=s["x_factor"], w1_global=s["w1_factor"], h_global=s["h_factor"], w2_global=s["w2_factor"])
        return s["y"]
    if kind == "quantise":
        v, scale = _quantise(s["x"], fmt, s["factor"])
        y = v.float() * _numbers(scale, fmt).repeat_interleave(_BLOCK[fmt], -1)[..., :case["cols"]]
        return {"y": (y if s["factor"] is None else y * s["factor"]).to(s["y"].dtype), "scale": scale.view(_SCALES[fmt])}
    if kind == "dequantise":
        y = _values(s["q"], s["scale"], fmt, case["cols"])
        return (y if s["factor"] is None else y * s["factor"]).to(s["y"].dtype)
    return _plain_matmul(s, case) if kind == "matmul" else _plain_experts(s, case)


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------

_BORDERS = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]  # between neighbouring 4-bit values; a tie goes up from the odd ones of them, else down


def _exact_quantise(x, fmt, factor):
    """(the numbers without the factor, their scales), in 64 bits: every element against the borders of its block."""
    cols, b = x.shape[1], _BLOCK[fmt]
    x = x.double()
    block = torch.arange(cols, device=x.device) // b
    amax = torch.zeros(x.shape[0], _blocks(cols, fmt), dtype=torch.float64, device=x.device)
    amax.scatter_reduce_(1, block.expand(x.shape[0], -1), x.abs(), "amax")
    g = torch.ones(1, dtype=torch.float64, device=x.device) if factor is None else factor.double()
    if fmt == "mx":
        powers = torch.ldexp(torch.ones(255, dtype=torch.float64, device=x.device), torch.arange(255, device=x.device) - 127)
        scale = powers[torch.searchsorted(6.0 * powers, amax).clamp_max(254)]
    else:
        table = torch.arange(127, dtype=torch.uint8, device=x.device).view(torch.float8_e4m3fn).double()  # 0 to 448
        want = amax / (6.0 * g)
        hi = torch.searchsorted(table, want).clamp_max(126)
        lo = (hi - 1).clamp_min(0)
        down, up = want - table[lo], table[hi] - want
        scale = torch.where((down < up) | ((down == up) & (lo % 2 == 0)), table[lo], table[hi])
    step = (scale * g)[:, block]
    a = x.abs()
    code = torch.zeros_like(x, dtype=torch.long)
    for i, t in enumerate(_BORDERS):
        code += (a >= t * step) if i % 2 else (a > t * step)
    v = torch.tensor(_VALUES[:8], dtype=torch.float64, device=x.device)[code]
    return torch.where(step > 0, torch.copysign(v, x), 0.0) * scale[:, block], scale


def _exact_values(q, scale, fmt):
    codes = torch.stack([q & 15, q >> 4], -1).reshape(q.shape[0], -1).long()
    v = torch.tensor(_VALUES, dtype=torch.float64, device=q.device)[codes]
    s = scale.contiguous().view(_SCALES[fmt]).float().double() if fmt == "nv" else torch.pow(2.0, scale.double() - 127.0)
    return v * s[:, torch.arange(codes.shape[1], device=q.device) // _BLOCK[fmt]]


def exact(case, seed):
    s = prepare(case, seed)
    fmt = case["format"]
    if case["kind"] == "quantise":
        y, scale = _exact_quantise(s["x"], fmt, s["factor"])
        return {"y": y if s["factor"] is None else y * s["factor"].double(), "scale": scale}
    if case["kind"] == "dequantise":
        cols = case["cols"]
        q = s["q"]
        codes = torch.stack([q & 15, q >> 4], -1).reshape(q.shape[0], -1)[:, :cols].long()
        y = torch.tensor(_VALUES, dtype=torch.float64, device="cuda")[codes]
        n = s["scale"].double()
        n = torch.pow(2.0, n - 127.0) if fmt == "mx" else s["scale"].contiguous().view(torch.float8_e4m3fn).double()
        y = y * n[:, torch.arange(cols, device="cuda") // _BLOCK[fmt]]
        return y if s["factor"] is None else y * s["factor"].double()
    if case["kind"] == "matmul":
        a = _exact_values(s["a"], s["a_scale"], fmt)
        if case["groups"] == 1:
            y = a @ _exact_values(s["b"], s["b_scale"], fmt).t()
            return y if s["alpha"] is None else y * s["alpha"].double()
        y = torch.zeros(case["rows"], case["n"], dtype=torch.float64, device="cuda")
        at = s["offsets"].tolist()
        for i in range(case["groups"]):
            if at[i + 1] > at[i]:
                part = a[at[i]:at[i + 1]] @ _exact_values(s["b"][i], s["b_scale"][i], fmt).t()
                y[at[i]:at[i + 1]] = part if s["alpha"] is None else part * s["alpha"][i].double()
        return y
    one = torch.ones(case["experts"], dtype=torch.float64, device="cuda")
    f = {n: s[n].double() if s[n] is not None else one for n in ("x_factor", "w1_factor", "h_factor", "w2_factor")}
    x = _exact_quantise(s["x"], fmt, s["x_factor"])[0] * f["x_factor"][0]
    y = torch.zeros(case["tokens"], case["hidden"], dtype=torch.float64, device="cuda")
    for e in range(case["experts"]):
        token, slot = (s["ids"] == e).nonzero(as_tuple=True)
        if not token.numel():
            continue
        gate, up = (f["w1_factor"][e] * (x[token] @ _exact_values(s["w1"][e, j], s["w1_scale"][e, j], fmt).t()) for j in (0, 1))
        h = _exact_quantise(gate * torch.sigmoid(gate) * up, fmt, s["h_factor"])[0] * f["h_factor"][0]
        part = f["w2_factor"][e] * (h @ _exact_values(s["w2"][e], s["w2_scale"][e], fmt).t())
        y.index_add_(0, token, part * s["weights"].double()[token, slot][:, None])
    return y
