"""Caches in 8 and 4 bits, selection by bounds and single tokens over them, from their definitions in Python numbers and 64 bits; no code of the
library, and no conversion of torch's to 8-bit types."""
from __future__ import annotations

import math
from fractions import Fraction

import torch

FORMATS = {"e4m3": dict(most=448.0, bits=3, least=-6, low=-117, high=119, bytes=32), "e2m1": dict(most=6.0, bits=1, least=0, low=-125, high=125, bytes=16)}


def number(fmt, code):
    """What a code stands for, by its bits."""
    if fmt == "e2m1":
        sign, e, m = code >> 3, (code >> 1) & 3, code & 1
        value = m * 0.5 if e == 0 else (1 + m / 2) * 2.0 ** (e - 1)
    else:
        sign, e, m = code >> 7, (code >> 3) & 15, code & 7
        value = math.nan if (e, m) == (15, 7) else m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
    return -value if sign else value


def group(fmt, values):
    """(scale byte, numbers) of up to 32 features: the least power of two under which none passes the largest number, then the nearest number, ties
    to the even code.  In exact fractions."""
    f = FORMATS[fmt]
    if not all(math.isfinite(v) for v in values):
        return 255, [math.nan] * len(values)
    amax, s = max(abs(v) for v in values), f["low"]
    while s < f["high"] and Fraction(amax) > Fraction(f["most"]) * Fraction(2) ** s:
        s += 1
    table = [number(fmt, c) for c in range(127 if fmt == "e4m3" else 8)]
    out = []
    for v in values:
        y = min(Fraction(abs(v)) / Fraction(2) ** s, Fraction(f["most"]))
        best = min(range(len(table)), key=lambda c: (abs(Fraction(table[c]) - y), c % 2))
        out.append(math.copysign(float(Fraction(table[best]) * Fraction(2) ** s), v))
    return s + 127, out


def stored(fmt, row):
    """(scale bytes, numbers) of a row of features."""
    scales, out = [], []
    for lo in range(0, len(row), 32):
        s, v = group(fmt, row[lo:lo + 32])
        scales.append(s)
        out += v
    return scales, out


def stored_rows(fmt, x):
    """Numbers of x [..., d], by rows, vectorised; the same as `stored` (tests compare the two)."""
    f, d = FORMATS[fmt], x.shape[-1]
    y = torch.nn.functional.pad(x.double(), (0, -d % 32)).unflatten(-1, (-1, 32))
    amax = y.abs().amax(-1, keepdim=True)
    finite = torch.isfinite(y).all(-1, keepdim=True)
    _, s = torch.frexp(torch.where(finite, amax, torch.ones_like(amax)) / f["most"])
    s = torch.where(amax == f["most"] * torch.ldexp(torch.ones_like(amax), s - 1), s - 1, s).clamp(f["low"], f["high"])
    z = torch.where(finite, torch.ldexp(y, -s), torch.zeros_like(y)).clamp(-f["most"], f["most"])
    _, e = torch.frexp(z)
    step = torch.ldexp(torch.ones_like(z), (e - 1).clamp(min=f["least"]) - f["bits"])
    z = torch.ldexp((z / step).round() * step, s.expand_as(z))
    return torch.where(finite, z, torch.full_like(z, math.nan)).flatten(-2)[..., :d]


def codes(fmt, code, scale):
    """Numbers of code bytes [width] under scale bytes [groups]."""
    out = []
    for g, s in enumerate(scale):
        part = code[g * FORMATS[fmt]["bytes"]:(g + 1) * FORMATS[fmt]["bytes"]]
        each = part if fmt == "e4m3" else [x for c in part for x in (c & 15, c >> 4)]
        out += [math.nan if s == 255 else number(fmt, c) * 2.0 ** (s - 127) for c in each]
    return out


def bounds(values, block):
    """(least, largest) [blocks, d] of keys [held, d]; NaN where a key of the block is NaN."""
    lo, hi = [], []
    for at in range(0, values.shape[0], block):
        part = values[at:at + block]
        nan = part.isnan().any(0)
        lo.append(torch.where(nan, math.nan, part.amin(0)))
        hi.append(torch.where(nan, math.nan, part.amax(0)))
    return torch.stack(lo), torch.stack(hi)


def select(q, lo, hi, held, block, keep, sink, recent):
    """Blocks (list of `keep`, -1 behind the last) for one KV head: q [group, d], lo / hi [blocks, d]."""
    count = -(-held // block)
    if count <= keep:
        return list(range(count)) + [-1] * (keep - count)
    score = []
    for i in range(count):
        best = None
        for row in q.double():
            s = float((row.clamp(min=0) * hi[i].double() + row.clamp(max=0) * lo[i].double()).sum())  # clamp keeps a NaN
            s = (1, 0.0) if math.isnan(s) else (0, s)
            best = s if best is None or s > best else best
        score.append(best)
    order = sorted(range(count), key=lambda i: (not (i < sink or i >= count - recent), -score[i][0], -score[i][1], i))
    return sorted(order[:keep])


def attend(q, k, v, at, *, scale, cap=0.0, slope=0.0, length=None):
    """One head: q [d], k / v [keys, d] in 64 bits, `at` the keys that are seen (a list, one may stand there twice).  Returns out, lse, the sum of
    |p v|, and a bound of the relative error of a probability."""
    d = v.shape[1]
    if not at:
        return torch.zeros(d, dtype=torch.float64), -math.inf, torch.zeros(d, dtype=torch.float64), 0.0
    idx = torch.tensor(at)
    s = scale * (k[idx] @ q.double())
    size = scale * (k[idx].abs() @ q.double().abs())
    if cap:
        s = cap * torch.tanh(s / cap)
    if slope:
        far = slope * (length - 1 - idx).double()
        s, size = s - far, size + far
    z = torch.logsumexp(s, 0)
    w = torch.exp(s - z)
    # a sum of d products, a few roundings of numbers up to that size, the maximum, and their exponential
    delta = 2.0 ** -21 * (float(size.max()) + abs(float(z)) + 4)
    return w @ v[idx], float(z), w @ v[idx].abs(), delta


def out_bound(out, out_abs, delta, dtype):
    """Probabilities are off by delta, relatively, sums of up to a few thousand terms by 2^-19; bf16 rounds the probabilities and the result, each by
    at most half a unit in the last place, 2^-8 of itself."""
    b = (2 * delta + 2.0 ** -19) * out_abs + 1e-30
    if dtype == torch.bfloat16:
        b = b + 2.0 ** -8 * out_abs + 2.0 ** -8 * out.abs()
    return b
