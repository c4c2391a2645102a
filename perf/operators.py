"""The operators of quantised linear and expert layers whose speed is measured.

Four kinds of case, all in 8-bit floating point with a scale for each block of 128:

* ``quantise``: a matrix to 8 bits, one scale for each 1 x 128 run of a row (activations) or 128 x 128 block (weights);
* ``matmul``: the product of two such matrices, alone or one for each group of consecutive rows (an expert's tokens);
* ``route``: which experts a token goes to, and with which weights;
* ``experts``: a gated feed-forward layer of routed experts, from the tokens and their routes to the layer's output.

The plain form is written with elementary torch operations in 32 bits (routing scores in 64, because neighbouring
scores decide which expert is taken), the other side is the package's own calls.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
_LARGEST = {"e4m3": 448.0, "e5m2": 57344.0}  # largest finite value of each 8-bit type
_SMALLEST_AMAX = 2.0 ** -100  # a block's largest magnitude counts as at least this much
_SIZE = {"f32": 4, "f16": 2, "bf16": 2}


# ---- cases -----------------------------------------------------------------------------------------------------------

def listed():
    return [
        # The activations of one token on their way into a linear layer: the smallest call.
        dict(name="quantise_rows_1x4096", kind="quantise", rows=1, cols=4096, block=1, x="bf16", q="e4m3"),
        # The activations of a long prompt or a large batch.
        dict(name="quantise_rows_16384x8192", kind="quantise", rows=16384, cols=8192, block=1, x="bf16", q="e4m3"),
        # A weight matrix with a last block that is not full on either side, when a model is loaded.
        dict(name="quantise_blocks_8200x5136", kind="quantise", rows=8200, cols=5136, block=128, x="f32", q="e4m3"),
        # One token through a linear layer: every weight is read for one row.
        dict(name="matmul_1x8192x8192", kind="matmul", rows=1, n=8192, k=8192, groups=1, a="e4m3", b="e4m3", y="bf16"),
        # A small batch of sequences decoded together, odd sizes.
        dict(name="matmul_37x5136x4112", kind="matmul", rows=37, n=5136, k=4112, groups=1, a="e4m3", b="e4m3", y="f16"),
        # A prompt of medium length.
        dict(name="matmul_2048x4096x4096", kind="matmul", rows=2048, n=4096, k=4096, groups=1, a="e4m3", b="e4m3", y="bf16"),
        # A long prompt through a large layer: bound by arithmetic.
        dict(name="matmul_8192x8192x8192", kind="matmul", rows=8192, n=8192, k=8192, groups=1, a="e4m3", b="e4m3", y="bf16"),
        # Rows sorted by expert, each expert with a weight matrix of its own; ragged groups, some empty.
        dict(name="matmul_8192x2048x4096_g32", kind="matmul", rows=8192, n=2048, k=4096, groups=32, a="e4m3", b="e4m3", y="bf16"),
        # One token's route.
        dict(name="route_1_of_64", kind="route", tokens=1, experts=64, topk=4, score="softmax", groups=1, topk_groups=1,
             group_score="max", bias=False, renormalise=True, scale=1.0, x="f32"),
        # The routes of a long prompt: sigmoid scores, a bias for balance, four of eight groups.
        dict(name="route_16384_of_256", kind="route", tokens=16384, experts=256, topk=8, score="sigmoid", groups=8, topk_groups=4,
             group_score="top2", bias=True, renormalise=True, scale=2.5, x="f32"),
        # A small batch decoded together through an expert layer: most experts' weights are read for a few rows each.
        dict(name="experts_16_of_64", kind="experts", tokens=16, experts=64, topk=4, hidden=2048, inter=1024, x="bf16"),
        # A long prompt through the same layer: bound by arithmetic.
        dict(name="experts_8192_of_64", kind="experts", tokens=8192, experts=64, topk=4, hidden=2048, inter=1024, x="bf16"),
    ]


def _log(rng, lo, hi):
    """An integer between lo and hi, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["quantise", "matmul", "matmul", "matmul", "route", "experts", "experts"])
    if kind == "quantise":
        cols = _log(rng, 100, 8192)
        if rng.random() < 0.5:
            cols = (cols + 15) // 16 * 16
        x = rng.choice(["bf16", "bf16", "f16", "f32"])
        most = min(16384, 400e6 / cols / (_SIZE[x] + 1))
        return dict(kind=kind, rows=_log(rng, 1, most), cols=cols, block=rng.choice([1, 1, 128]), x=x,
                    q=rng.choice(["e4m3", "e4m3", "e4m3", "e5m2"]))
    if kind == "matmul":
        groups = rng.choice([1, 1, 1, rng.randint(2, 64)])
        n, k = _log(rng, 64, 8192), 16 * _log(rng, 8, 512)
        if rng.random() < 0.5:
            n = (n + 63) // 64 * 64
        if groups > 1:
            n, k = min(n, 4096), min(k, 4096)
            groups = min(groups, max(2, (1 << 28) // (n * k)))
        return dict(kind=kind, rows=_log(rng, 1, 8192), n=n, k=k, groups=groups, a=rng.choice(["e4m3", "e4m3", "e4m3", "e5m2"]),
                    b="e4m3", y=rng.choice(["bf16", "bf16", "f16", "f32"]))
    if kind == "route":
        experts = rng.choice([8, 16, 60, 64, 96, 128, 160, 256, 512])
        groups = rng.choice([1, 1, 4, 8]) if experts % 8 == 0 and experts >= 32 else 1
        topk_groups = rng.randint(1, groups)
        return dict(kind=kind, tokens=_log(rng, 1, 16384), experts=experts, topk=rng.randint(1, min(8, experts // groups)),
                    score=rng.choice(["softmax", "sigmoid"]), groups=groups, topk_groups=topk_groups,
                    group_score=rng.choice(["max", "top2"]), bias=rng.random() < 0.5, renormalise=rng.random() < 0.7,
                    scale=rng.choice([1.0, 2.5]), x=rng.choice(["f32", "bf16"]))
    experts = rng.choice([8, 16, 24, 32, 64])
    return dict(kind=kind, tokens=_log(rng, 1, 8192), experts=experts, topk=rng.randint(1, 4), hidden=16 * _log(rng, 16, 128),
                inter=16 * _log(rng, 8, 64), x=rng.choice(["bf16", "bf16", "f16"]))


def _blocks(n):
    return (n + 127) // 128


def _active(tokens, experts, topk):
    """Expected number of experts that get a token, each token taking `topk` different ones."""
    return experts * (1.0 - (1.0 - topk / experts) ** tokens)


def work(case):
    c = case
    if c["kind"] == "quantise":
        scales = -(-c["rows"] // c["block"]) * _blocks(c["cols"])
        return {"bytes": c["rows"] * c["cols"] * (_SIZE[c["x"]] + 1) + 4 * scales, "flops": 2 * c["rows"] * c["cols"]}
    if c["kind"] == "matmul":
        rows = c["rows"] - (c["rows"] // 16 if c["groups"] > 1 else 0)  # the rest belongs to no group
        weights = 1 if c["groups"] == 1 else max(1, min(c["groups"] - 1, rows))
        return {"bytes": rows * (c["k"] + 4 * _blocks(c["k"]) + c["n"] * _SIZE[c["y"]]) + weights * c["n"] * c["k"],
                "flops": 2 * rows * c["n"] * c["k"]}
    if c["kind"] == "route":
        return {"bytes": c["tokens"] * (c["experts"] * _SIZE[c["x"]] + 8 * c["topk"]), "flops": c["tokens"] * c["experts"] * 8}
    matrix = c["hidden"] * c["inter"]
    return {"bytes": 3 * matrix * _active(c["tokens"], c["experts"], c["topk"]) + c["tokens"] * (2 * c["hidden"] * _SIZE[c["x"]] + 8 * c["topk"]),
            "flops": 6 * matrix * c["tokens"] * c["topk"]}


# ---- plain forms -----------------------------------------------------------------------------------------------------

def _pad(x, *multiples):
    """`x` with zeros behind its last axes, up to the given multiples."""
    sizes = []
    sizes += [v for n, m in reversed(list(zip(x.shape[-len(multiples):], multiples))) for v in (0, -n % m)]
    return torch.nn.functional.pad(x, sizes) if any(sizes) else x


def _quantise(x, block, q):
    """(8-bit values, scales) of a matrix or of a stack of matrices."""
    rows, cols = x.shape[-2:]
    p = _pad(x.float(), block, 128)
    p = p.reshape(*x.shape[:-2], p.shape[-2] // block, block, p.shape[-1] // 128, 128)
    amax = p.abs().amax(dim=(-3, -1), keepdim=True).clamp_min(_SMALLEST_AMAX)
    v = (p * _LARGEST[q] / amax).to(_TYPES[q])  # (one product, exact for 16-bit inputs, one division: a tie stays a tie)
    v = v.view(torch.uint8).reshape(*x.shape[:-2], p.shape[-4] * block, p.shape[-2] * 128)[..., :rows, :cols].contiguous().view(_TYPES[q])
    return v, (amax / _LARGEST[q]).squeeze(-1).squeeze(-2).contiguous()


def _values(q, scale, block):
    """The numbers that 8-bit values and their scales stand for, in 32 bits."""
    rows, cols = q.shape[-2:]
    s = scale.repeat_interleave(block, -2)[..., :rows, :] if block > 1 else scale
    return q.float() * s.repeat_interleave(128, -1)[..., :cols]


def _plain_matmul(s, case):
    a, b = _values(s["a"], s["a_scale"], 1), _values(s["b"], s["b_scale"], 128)
    if case["groups"] == 1:
        return torch.matmul(a, b.t()).to(s["y"].dtype)
    first, count = s["offsets"][:-1].long(), (s["offsets"][1:] - s["offsets"][:-1]).long()
    at = torch.arange(s["most"], device=a.device)
    index = (first[:, None] + at).clamp_max(a.shape[0] - 1)
    y = torch.matmul(a[index], b.transpose(-1, -2))
    out = torch.zeros(a.shape[0] + 1, case["n"], device=a.device)  # (the last row takes what no group has)
    out[torch.where(at < count[:, None], index, a.shape[0])] = y
    return out[:-1].to(s["y"].dtype)


def _plain_route(s, case):
    x = s["logits"].double()
    if case["score"] == "softmax":
        e = torch.exp(x - x.amax(-1, keepdim=True))
        score = e / e.sum(-1, keepdim=True)
    else:
        score = 1.0 / (1.0 + torch.exp(-x))
    choice = score + s["bias"].double() if case["bias"] else score
    if case["groups"] > 1:
        by = choice.reshape(x.shape[0], case["groups"], -1)
        best = by.amax(-1) if case["group_score"] == "max" else by.sort(-1, descending=True).values[..., :2].sum(-1)
        kept = best.sort(dim=-1, descending=True, stable=True).indices[:, :case["topk_groups"]]
        mask = torch.zeros_like(best, dtype=torch.bool).scatter(1, kept, True)
        choice = torch.where(mask[:, :, None], by, -math.inf).reshape(x.shape)
    ids = choice.sort(dim=-1, descending=True, stable=True).indices[:, :case["topk"]]
    w = score.gather(1, ids)
    if case["renormalise"]:
        w = w / w.sum(-1, keepdim=True)
    return (w * case["scale"]).float(), ids.int()


def _gated(h):
    gate, up = h.chunk(2, -1)
    return gate / (1.0 + torch.exp(-gate)) * up


def _plain_experts(s, case):
    T, K, E, H, I = case["tokens"], case["topk"], case["experts"], case["hidden"], case["inter"]
    x = _values(*_quantise(s["x"], 1, "e4m3"), 1)
    ids = s["ids"].long()
    if T * K <= E:  # few rows: each with its own expert's matrices
        w1 = _values(s["w1"][ids.reshape(-1)], s["w1_scale"][ids.reshape(-1)], 128).reshape(T * K, 2 * I, H)
        w2 = _values(s["w2"][ids.reshape(-1)], s["w2_scale"][ids.reshape(-1)], 128)
        h = _gated(torch.matmul(w1, x.repeat_interleave(K, 0)[:, :, None]).squeeze(-1))
        h = _values(*_quantise(h, 1, "e4m3"), 1)
        y = torch.matmul(w2, h[:, :, None]).squeeze(-1).reshape(T, K, H)
    else:  # all experts at once, each expert's rows padded to the longest
        w1 = _values(s["w1"], s["w1_scale"], 128).reshape(E, 2 * I, H)
        w2 = _values(s["w2"], s["w2_scale"], 128)
        chosen = torch.zeros(T, E, dtype=torch.long, device=x.device).scatter(1, ids, 1)
        place = (chosen.cumsum(0) - chosen).gather(1, ids)  # how many earlier tokens took the same expert
        rows = torch.zeros(E, s["most"], H, device=x.device)
        rows[ids, place] = x[:, None, :].expand(T, K, H)
        h = _gated(torch.matmul(rows, w1.transpose(1, 2)))
        h = _values(*_quantise(h, 1, "e4m3"), 1)
        y = torch.matmul(h, w2.transpose(1, 2))[ids, place]
    return (y * s["weights"][:, :, None]).sum(1).to(s["y"].dtype)


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _activations(g, *shape):
    """Normal values, one column in about five hundred twenty times larger, as hidden states have them."""
    big = torch.rand(shape[-1], generator=g, device="cuda") < 0.002
    return torch.randn(*shape, generator=g, device="cuda") * torch.where(big, 20.0, 1.0)


def _weights(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda") / math.sqrt(shape[-1])


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = {"case": dict(case)}
    if case["kind"] == "quantise":
        rows, cols = case["rows"], case["cols"]
        s["x"] = (_activations(g, rows, cols) if case["block"] == 1 else _weights(g, rows, cols)).to(_TYPES[case["x"]])
        s["q"] = torch.zeros(rows, cols, dtype=torch.uint8, device="cuda").view(_TYPES[case["q"]])
        s["scale"] = torch.zeros(-(-rows // case["block"]), _blocks(cols), device="cuda")
    elif case["kind"] == "matmul":
        rows, n, k, groups = case["rows"], case["n"], case["k"], case["groups"]
        s["a"], s["a_scale"] = _quantise(_activations(g, rows, k), 1, case["a"])
        s["b"], s["b_scale"] = _quantise(_weights(g, *([groups] if groups > 1 else []), n, k), 128, case["b"])
        s["y"] = torch.zeros(rows, n, dtype=_TYPES[case["y"]], device="cuda")
        s["offsets"], s["most"] = None, 0
        if groups > 1:  # uneven groups, one of them empty, and a few rows behind the last one
            share = torch.exp(0.7 * torch.randn(groups, generator=g, device="cuda"))
            share[torch.randint(groups, (1,), generator=g, device="cuda")] = 0.0
            of = torch.multinomial(share, rows - rows // 16, replacement=True, generator=g)
            count = torch.bincount(of, minlength=groups)
            s["offsets"] = torch.nn.functional.pad(count.cumsum(0), (1, 0)).int()
            s["most"] = int(count.max())
    elif case["kind"] == "route":
        x = torch.randn(case["tokens"], case["experts"], generator=g, device="cuda") * 1.5
        s["logits"] = x.to(_TYPES[case["x"]])
        s["bias"] = torch.randn(case["experts"], generator=g, device="cuda") * 0.05 if case["bias"] else None
        s["weights"] = torch.zeros(case["tokens"], case["topk"], device="cuda")
        s["ids"] = torch.zeros(case["tokens"], case["topk"], dtype=torch.int32, device="cuda")
    else:
        T, K, E, H, I = case["tokens"], case["topk"], case["experts"], case["hidden"], case["inter"]
        s["x"] = _activations(g, T, H).to(_TYPES[case["x"]])
        s["w1"], s["w1_scale"] = _quantise(_weights(g, E, 2, I, H), 128, "e4m3")  # gate, then up
        s["w2"], s["w2_scale"] = _quantise(_weights(g, E, H, I), 128, "e4m3")
        score = torch.rand(T, E, generator=g, device="cuda") + 0.2 * torch.rand(E, generator=g, device="cuda")
        top = score.topk(K, -1)
        s["ids"], s["weights"] = top.indices.int(), top.values / top.values.sum(-1, keepdim=True)
        s["y"] = torch.zeros(T, H, dtype=_TYPES[case["x"]], device="cuda")
        s["most"] = int(torch.bincount(s["ids"].reshape(-1), minlength=E).max())
    return s


# ---- one pass --------------------------------------------------------------------------------------------------------

def run(state):
    s, case = state, state["case"]
    if own:
        import paper_2104_04731_b200 as b2c

        if case["kind"] == "quantise":
            b2c.fp8_quantize(s["x"], s["q"], s["scale"], block_rows=case["block"])
            return {"q": s["q"], "scale": s["scale"]}
        if case["kind"] == "matmul":
            b2c.fp8_matmul(s["a"], s["a_scale"], s["b"], s["b_scale"], s["y"], offsets=s["offsets"])
            return s["y"]
        if case["kind"] == "route":
            if "desc" not in s:
                s["desc"] = b2c.make_route_desc(
                    case["experts"], case["topk"], score=b2c.SCORE_SOFTMAX if case["score"] == "softmax" else b2c.SCORE_SIGMOID,
                    groups=case["groups"], topk_groups=case["topk_groups"],
                    group_score=b2c.GROUP_MAX if case["group_score"] == "max" else b2c.GROUP_TOP2,
                    renormalise=case["renormalise"], scale=case["scale"])
            b2c.route(s["desc"], s["logits"], s["weights"], s["ids"], bias=s["bias"])
            return {"weights": s["weights"], "ids": s["ids"]}
        if "workspace" not in s:
            n = b2c.experts_workspace_bytes(case["hidden"], case["inter"], case["experts"], case["topk"], case["tokens"])
            s["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
        b2c.fp8_experts(s["x"], s["ids"], s["weights"], s["w1"], s["w1_scale"], s["w2"], s["w2_scale"], s["y"], s["workspace"])
        return s["y"]
    if case["kind"] == "quantise":
        q, scale = _quantise(s["x"], case["block"], case["q"])
        return {"q": q, "scale": scale}
    if case["kind"] == "matmul":
        return _plain_matmul(s, case)
    if case["kind"] == "route":
        w, ids = _plain_route(s, case)
        return {"weights": w, "ids": ids}
    return _plain_experts(s, case)


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------

def _round8(v, q):
    """The nearest value of an 8-bit type (ties to even), |v| within its largest: steps of 2^(exponent - mantissa bits)."""
    mantissa, lowest = (3, -6) if q == "e4m3" else (2, -14)
    _, e = torch.frexp(v)  # |v| in [2^(e-1), 2^e)
    step = torch.ldexp(torch.ones_like(v), (e - 1).clamp_min(lowest) - mantissa)
    return torch.round(v / step) * step


def _exact_quantise(x, block, q):
    rows, cols = x.shape
    row_block = torch.arange(rows, device=x.device) // block
    col_block = torch.arange(cols, device=x.device) // 128
    amax = torch.zeros(-(-rows // block), _blocks(cols), dtype=torch.float64, device=x.device)
    x = x.double()
    index = row_block[:, None] * amax.shape[1] + col_block
    amax.view(-1).scatter_reduce_(0, index.reshape(-1), x.abs().reshape(-1), "amax")
    amax = amax.clamp_min(_SMALLEST_AMAX)
    return _round8(x * _LARGEST[q] / amax[row_block][:, col_block], q), amax / _LARGEST[q]


def _exact_values(q, scale, block):
    r = torch.arange(q.shape[0], device=q.device) // block
    c = torch.arange(q.shape[1], device=q.device) // 128
    return q.double() * scale.double()[r][:, c]


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "quantise":
        q, scale = _exact_quantise(s["x"], case["block"], case["q"])
        return {"q": q, "scale": scale}
    if case["kind"] == "matmul":
        a = _exact_values(s["a"], s["a_scale"], 1)
        if case["groups"] == 1:
            return a @ _exact_values(s["b"], s["b_scale"], 128).t()
        y = torch.zeros(case["rows"], case["n"], dtype=torch.float64, device="cuda")
        at = s["offsets"].tolist()
        for g in range(case["groups"]):
            if at[g + 1] > at[g]:
                y[at[g]:at[g + 1]] = a[at[g]:at[g + 1]] @ _exact_values(s["b"][g], s["b_scale"][g], 128).t()
        return y
    if case["kind"] == "route":
        x = s["logits"].double()
        score = torch.softmax(x, -1) if case["score"] == "softmax" else torch.sigmoid(x)
        choice = score + (s["bias"].double() if case["bias"] else 0.0)
        taken = torch.zeros_like(choice, dtype=torch.bool)
        size = case["experts"] // case["groups"]
        if case["groups"] > 1:
            parts = choice.split(size, -1)
            value = torch.stack([p.amax(-1) if case["group_score"] == "max" or size == 1 else p.topk(2, -1).values.sum(-1) for p in parts], -1)
            open_ = torch.zeros_like(value, dtype=torch.bool)
            for _ in range(case["topk_groups"]):
                best = torch.where(open_, -math.inf, value).max(-1, keepdim=True).values
                first = ((value == best) & ~open_).int().argmax(-1, keepdim=True)
                open_.scatter_(1, first, True)
            taken |= ~open_.repeat_interleave(size, -1)
        ids = []
        for _ in range(case["topk"]):
            best = torch.where(taken, -math.inf, choice).max(-1, keepdim=True).values
            first = ((choice == best) & ~taken).int().argmax(-1, keepdim=True)
            taken = taken.scatter(1, first, True)
            ids.append(first)
        ids = torch.cat(ids, -1)
        w = score.gather(1, ids)
        w = w / w.sum(-1, keepdim=True) if case["renormalise"] else w
        return {"weights": w * case["scale"], "ids": ids.int()}
    x = _exact_quantise(s["x"], 1, "e4m3")
    c = torch.arange(case["hidden"], device="cuda") // 128
    x = x[0] * x[1][:, c]
    y = torch.zeros(case["tokens"], case["hidden"], dtype=torch.float64, device="cuda")
    for e in range(case["experts"]):
        token, slot = (s["ids"] == e).nonzero(as_tuple=True)
        if not token.numel():
            continue
        gate, up = (x[token] @ _exact_values(s["w1"][e, j], s["w1_scale"][e, j], 128).t() for j in (0, 1))
        h, scale = _exact_quantise(gate * torch.sigmoid(gate) * up, 1, "e4m3")
        h = h * scale[:, torch.arange(case["inter"], device="cuda") // 128]
        part = h @ _exact_values(s["w2"][e], s["w2_scale"][e], 128).t()
        y.index_add_(0, token, part * s["weights"].double()[token, slot][:, None])
    return y
