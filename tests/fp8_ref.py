"""The 8-bit float operators written out in 64 bits with torch, for the tests; shares no code with the library."""
import math

import torch

LARGEST = {torch.float8_e4m3fn: 448.0, torch.float8_e5m2: 57344.0}
MANTISSA = {torch.float8_e4m3fn: 3, torch.float8_e5m2: 2}
LOWEST = {torch.float8_e4m3fn: -6, torch.float8_e5m2: -14}


def nb(n):
    return -(-n // 128)


def round8(v, dtype):
    """Nearest value of an 8-bit type, ties to even, of |v| up to its largest; NaN stays."""
    _, e = torch.frexp(torch.where(v.isnan(), 1.0, v))
    step = torch.ldexp(torch.ones_like(v), (e - 1).clamp_min(LOWEST[dtype]) - MANTISSA[dtype])
    return (torch.round(v / step) * step).clamp(-LARGEST[dtype], LARGEST[dtype])


def spread(scale, rows, cols, block_rows):
    """One scale for every element."""
    dev = scale.device
    return scale.double()[torch.arange(rows, device=dev) // block_rows][:, torch.arange(cols, device=dev) // 128]


def amax_of(x, block_rows):
    rows, cols = x.shape
    v = torch.zeros(-(-rows // block_rows) * block_rows, nb(cols) * 128, dtype=torch.float64, device=x.device)
    v[:rows, :cols] = torch.nan_to_num(x.double().abs(), nan=0.0, posinf=math.inf)
    return v.reshape(-1, block_rows, nb(cols), 128).amax((1, 3)).clamp_min(2.0 ** -100)


def quantize(x, dtype, block_rows=1):
    """(values, scale), both in 64 bits."""
    rows, cols = x.shape
    amax = amax_of(x, block_rows)
    a = spread(amax, rows, cols, block_rows)
    v = torch.where(a.isinf(), torch.where(x.double().isinf(), math.nan, 0.0 * x.double()), x.double() * LARGEST[dtype] / a)
    return round8(v, dtype), amax / LARGEST[dtype]


def values(q, scale, block_rows):
    return q.double() * spread(scale, q.shape[0], q.shape[1], block_rows)


def matmul(a, a_scale, b, b_scale):
    return values(a, a_scale, 1) @ values(b, b_scale, 128).t()


def size_of_sums(a, a_scale, b, b_scale):
    """Sum of the magnitudes of every output's products: what rounding errors of the sums are relative to."""
    return values(a, a_scale, 1).abs() @ values(b, b_scale, 128).abs().t()


def sum_error(K):
    """Relative error of a sum of K products scaled in blocks of 128, fp32, any order.  Products of 8-bit values are exact; a sum of n terms is
    off by at most (n - 1) units of rounding (2^-23 where partial sums are cut off instead of rounded), the scaled addition of every block by
    three more (product of the scales, product with the block's sum, addition)."""
    return (K + 3 * nb(K)) * 2.0 ** -23


def scores(logits, kind):
    x = logits.double()
    x = torch.where(x.isnan(), -math.inf, x)
    if kind == "sigmoid":
        return torch.where(x == -math.inf, 0.0, 1 / (1 + torch.exp(-x)))
    m = x.amax(-1, keepdim=True)
    e = torch.where(x == -math.inf, 0.0, torch.where(x == m, 1.0, torch.exp(x - torch.where(m.isinf(), 0.0, m))))
    e = torch.where((m == math.inf) & (x != m), 0.0, e)
    s = e.sum(-1, keepdim=True)
    return torch.where(s > 0, e / torch.where(s > 0, s, 1.0), 0.0)


def route(logits, topk, kind="softmax", groups=1, topk_groups=1, group_score="max", renormalise=True, scale=1.0, bias=None):
    """Plain loops over the tokens of a small batch: (weights in 64 bits, ids)."""
    s = scores(logits, kind).cpu()
    part = s + (bias.double().cpu() if bias is not None else 0.0)
    # scores are monotonic in the logits: without a bias these decide, and a run's largest choice is that of its largest logit
    choice = part if bias is not None else logits.double().cpu()
    if bias is None and group_score == "max":
        part = choice
    ids, weights = [], []
    for t in range(s.shape[0]):
        c, of_run = ([v if v == v else -math.inf for v in x[t].tolist()] for x in (choice, part))
        size = len(c) // groups
        runs = []
        for g in range(groups):
            top = sorted(of_run[g * size:(g + 1) * size], reverse=True)
            score = top[0] if group_score == "max" or size == 1 else top[0] + top[1]
            runs.append((-score if score == score else math.inf, g))
        kept = {g for _, g in sorted(runs)[:topk_groups]}
        chosen = sorted((-c[e], e) for e in range(len(c)) if e // size in kept)[:topk]
        chosen = [e for _, e in chosen]
        w = s[t, chosen]
        if renormalise:
            w = w / w.sum() if w.sum() > 0 else w * 0
        ids.append(chosen)
        weights.append(w * scale)
    if not ids:
        return torch.zeros(0, topk, dtype=torch.float64), torch.zeros(0, topk, dtype=torch.int32)
    return torch.stack(weights), torch.tensor(ids, dtype=torch.int32)


def sort(ids, experts):
    """(offsets, rows, order) of the stable sort of the pairs by expert."""
    flat = ids.reshape(-1).cpu()
    order = [p for e in range(experts) for p in (flat == e).nonzero().flatten().tolist()]
    offsets = [0]
    for e in range(experts):
        offsets.append(offsets[-1] + int((flat == e).sum()))
    rows = torch.full((flat.numel(),), -1, dtype=torch.int32)
    for at, p in enumerate(order):
        rows[p] = at
    return torch.tensor(offsets, dtype=torch.int32), rows, torch.tensor(order, dtype=torch.int32)


def experts(x, ids, weights, w1, w1_scale, w2, w2_scale, out_dtype):
    """(y in 64 bits, a bound on the error of every element).

    The bound follows the rounding errors: a value h of the gated product is off by the errors of its two sums, of the
    logistic function and of two products; where that moves it across the border between two 8-bit values, its
    quantised value moves by a step.  Both ends of h's interval are quantised, and the difference goes through the second
    product; then come that product's own error, the rounding of its row and of the weighted sum."""
    T, K = ids.shape
    half = torch.finfo(out_dtype).eps / 2
    y = torch.zeros(T, x.shape[1], dtype=torch.float64, device=x.device)
    err = torch.zeros_like(y)
    xq, xs = quantize(x, torch.float8_e4m3fn)
    for e in range(w1.shape[0]):
        token, slot = (ids == e).nonzero(as_tuple=True)
        if not token.numel():
            continue
        xe, se = xq[token], xs[token].float()
        H, I = x.shape[1], w1.shape[2]
        gate, up = (matmul(xe, se, w1[e, j], w1_scale[e, j]) for j in (0, 1))
        dg, du = (sum_error(H) * size_of_sums(xe, se, w1[e, j], w1_scale[e, j]) for j in (0, 1))
        sg = gate * torch.sigmoid(gate)
        h = sg * up
        # |silu'| <= 1.1; the logistic function in fp32 is off by a few units (8 taken), the products by one each
        dh = 1.1 * dg * up.abs() + (sg.abs() + 1.1 * dg) * du + 10 * 2.0 ** -24 * h.abs()
        amax = amax_of(h, 1)
        damax = amax_of(dh, 1)  # the largest magnitude moves by at most the largest error
        a, da = spread(amax, h.shape[0], I, 1), spread(damax, h.shape[0], I, 1)
        mid = round8(h * 448 / a, torch.float8_e4m3fn) * a / 448
        ends = [round8((h + s * dh) * 448 / (a + u * da).clamp_min(2.0 ** -100), torch.float8_e4m3fn) * (a + u * da) / 448 for s in (-1, 1) for u in (-1, 1)]
        dq = torch.stack([(v - mid).abs() for v in ends]).amax(0) + 2.0 ** -23 * mid.abs()
        w = values(w2[e], w2_scale[e], 128)
        part = mid @ w.t()
        dpart = dq @ w.abs().t() + sum_error(I) * ((mid.abs() + dq) @ w.abs().t())
        dpart = dpart + half * (part.abs() + dpart)
        wt = weights.double()[token, slot][:, None]
        y.index_add_(0, token, part * wt)
        err.index_add_(0, token, dpart * wt.abs() + 2.0 ** -23 * K * (part.abs() + dpart) * wt.abs())
    return y, err + half * (y.abs() + err) + 2.0 ** -24 * torch.finfo(out_dtype).smallest_normal
