"""The 4-bit float operators written out in 64 bits with torch, for the tests; shares no code with the library."""
import math

import torch

MX, NV = 0, 1
BLOCK = {MX: 32, NV: 16}
SCALE = {MX: torch.float8_e8m0fnu, NV: torch.float8_e4m3fn}
VALUES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def nb(n, fmt):
    return -(-n // BLOCK[fmt])


def spread(scale, cols, fmt):
    """One scale for every element."""
    return scale[..., torch.arange(cols, device=scale.device) // BLOCK[fmt]]


# (tables by Python's numbers: torch's powers of two on the device are not exact)
NUMBERS = {MX: [2.0 ** (c - 127) for c in range(255)] + [math.nan],
           NV: [(c % 8) / 8 * 2.0 ** -6 if c < 8 else (1 + (c % 8) / 8) * 2.0 ** (c // 8 - 7) for c in range(127)] + [math.nan] * 129}


def scale_numbers(scale, fmt):
    """Stored scales as numbers, by their definition."""
    return torch.tensor(NUMBERS[fmt], dtype=torch.float64, device=scale.device)[scale.contiguous().view(torch.uint8).long()]


def unpack(q, cols):
    q = q.view(torch.uint8)
    code = torch.stack([q & 15, q >> 4], -1).reshape(*q.shape[:-1], -1)[..., :cols]
    v = torch.tensor(VALUES, dtype=torch.float64, device=q.device)[(code & 7).long()]
    return torch.where(code > 7, -v, v)


def pack(code):
    """Codes (0..15) of a matrix with an even number of columns, packed."""
    return (code[..., 0::2] | (code[..., 1::2] << 4)).to(torch.uint8)


def values(q, scale, fmt, cols=None):
    cols = 2 * q.shape[-1] if cols is None else cols
    return unpack(q, cols) * spread(scale_numbers(scale, fmt), cols, fmt)


def round4(a):
    """Nearest of the 4-bit values, ties to the even code, of magnitudes; 6 beyond."""
    v = torch.tensor(VALUES, dtype=torch.float64, device=a.device)
    code = torch.zeros(a.shape, dtype=torch.long, device=a.device)
    for i in range(7):
        mid = (v[i] + v[i + 1]) / 2
        code += (a >= mid) if i % 2 else (a > mid)
    return v[code]


def e4m3(a):
    """Nearest E4M3 value, ties to even, of magnitudes; 448 beyond."""
    _, e = torch.frexp(a)
    step = torch.ldexp(torch.ones_like(a), (e - 1).clamp_min(-6) - 3)
    return (torch.round(a / step) * step).clamp_max(448.0)


def block_amax(x, fmt):
    rows, cols = x.shape
    v = torch.nn.functional.pad(x.double().abs(), (0, -cols % BLOCK[fmt]))
    return v.reshape(rows, nb(cols, fmt), BLOCK[fmt]).amax(-1)  # (a NaN makes its block's NaN)


def scales_of(amax, fmt, g=1.0):
    """Scales as numbers; NaN where amax is not finite."""
    fine = amax.isfinite()
    a = torch.where(fine, amax, 1.0)
    if fmt == MX:
        m, e = torch.frexp(a)
        e = torch.where(m <= 0.75, e - 3, e - 2)
        s = torch.ldexp(torch.ones_like(a), torch.where(a > 0, e, -127).clamp(-127, 127))
    else:
        s = e4m3(a / torch.full_like(a, 6 * g))  # (by a number torch divides on the device as by its reciprocal)
    return torch.where(fine, s, math.nan)


def rounded(x, scale, fmt, g=1.0):
    """The 4-bit values of x under these scales."""
    step = spread(scale, x.shape[1], fmt) * g
    on = step > 0  # (not NaN either)
    v = round4(torch.where(on, x.double().abs() / torch.where(on, step, 1.0), 0.0).nan_to_num(0.0))
    return torch.copysign(v, x.double().nan_to_num(0.0))


def quantize(x, fmt, g=None):
    """(4-bit values, scales), both in 64 bits."""
    g = 1.0 if g is None else float(g)
    s = scales_of(block_amax(x, fmt), fmt, g)
    return rounded(x, s, fmt, g), s


def sum_error(K):
    """Relative error of a sum of K scaled products in fp32, in any order: products of two values and two scales have 4 + 8 bits at most and are
    exact; a sum of n terms is off by at most (n - 1) units of rounding, 2^-23 where partial sums are cut off instead of rounded; one more
    for the factor."""
    return (K + 2) * 2.0 ** -23


def experts(x, ids, weights, w1, s1, w2, s2, fmt, out_dtype, gx=1.0, g1=None, gh=1.0, g2=None):
    """(y in 64 bits, a bound on the error of every element).

    The bound follows the rounding errors: a value h of the gated product is off by the errors of its two sums, of the logistic function and of
    the products; where that moves it, or its block's scale, across a border its quantised value moves.  Both ends of every interval are
    quantised and the difference goes through the second product; then come that product's own error and those of the weighted sum."""
    T, K = ids.shape
    n, H, I = w1.shape[0], x.shape[1], w1.shape[2]
    half = torch.finfo(out_dtype).eps / 2
    one = torch.ones(n, dtype=torch.float64, device=x.device)
    g1, g2 = (one if g is None else g.double() for g in (g1, g2))
    y = torch.zeros(T, H, dtype=torch.float64, device=x.device)
    err = torch.zeros_like(y)
    xq, xs = quantize(x, fmt, gx)
    xq = xq * spread(xs, H, fmt)
    for e in range(n):
        token, slot = (ids == e).nonzero(as_tuple=True)
        if not token.numel():
            continue
        f1 = float(g1[e]) * gx
        gate, up = (f1 * (xq[token] @ values(w1[e, j], s1[e, j], fmt).t()) for j in (0, 1))
        dg, du = ((sum_error(H) + 2.0 ** -23) * abs(f1) * (xq[token].abs() @ values(w1[e, j], s1[e, j], fmt).abs().t()) for j in (0, 1))
        sg = gate * torch.sigmoid(gate)
        h = sg * up
        # |silu'| <= 1.1.  In units of 2^-24 of h: 8 for the logistic function (its power, sum, reciprocal), 2 for the products with it and with
        # up, 3 for the quotient of the quantisation (step, its reciprocal, product); and 1.1 |gate| for the rounded exponent of e^-|gate|, which
        # is a relative error of that power and for negative gates of silu itself
        dh = 1.1 * dg * up.abs() + (sg.abs() + 1.1 * dg) * du + (13 + 1.1 * gate.abs()) * 2.0 ** -24 * h.abs()
        amax, damax = block_amax(h, fmt), block_amax(dh, fmt)
        scale = scales_of(amax, fmt, gh)
        mid = rounded(h, scale, fmt, gh) * spread(scale, I, fmt) * gh
        dq = torch.zeros_like(mid)
        for u in (-1, 1):
            other = scales_of((amax + u * (damax + 3 * 2.0 ** -24 * amax)).clamp_min(0.0), fmt, gh)
            for s in (scale, other):
                for d in (-1, 0, 1):
                    dq = torch.maximum(dq, (rounded(h + d * dh, s, fmt, gh) * spread(s, I, fmt) * gh - mid).abs())
        f2 = float(g2[e])
        w = f2 * values(w2[e], s2[e], fmt)
        part = mid @ w.t()
        dpart = dq @ w.abs().t() + (sum_error(I) + 2.0 ** -23) * ((mid.abs() + dq) @ w.abs().t())
        wt = weights.double()[token, slot][:, None]
        y.index_add_(0, token, part * wt)
        err.index_add_(0, token, dpart * wt.abs() + 2.0 ** -23 * K * (part.abs() + dpart) * wt.abs())
    return y, err + half * (y.abs() + err) + 2.0 ** -24 * torch.finfo(out_dtype).smallest_normal
