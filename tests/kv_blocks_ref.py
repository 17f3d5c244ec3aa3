"""Plain float64 forms of the operators on a cache cut into blocks, on the CPU: a cache's contents from whole sequences,
scores and selections of blocks, and attention over a selection.  Written from the definitions in include/a2ats.h."""
import math

import torch

D = 128
TINY = 2.0 ** -100


def e4m3_values():
    """All finite OCP e4m3 values >= 0 in order: 4 exponent bits (bias 7), 3 mantissa bits, 0x7f is the NaN."""
    out = []
    for code in range(0x7f):
        e, m = code >> 3, code & 7
        out.append(m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return torch.tensor(out, dtype=torch.float64)


_E4M3 = e4m3_values()


def round_e4m3(x):
    """Nearest e4m3 value of |x| <= 448, ties to the even code; returns (value with sign, code byte)."""
    a = x.abs()
    hi = torch.searchsorted(_E4M3, a.contiguous()).clamp(max=len(_E4M3) - 1)
    lo = (hi - 1).clamp(min=0)
    up, down = _E4M3[hi] - a, a - _E4M3[lo]
    take_hi = (up < down) | ((up == down) & (hi % 2 == 0))
    code = torch.where(take_hi, hi, lo)
    code = torch.where(_E4M3[hi] == a, hi, code)
    return torch.sign(x) * _E4M3[code], code


def quantise(x, fmt):
    """One block x [blk, D] (float64) -> (codes as the numbers they are, scale)."""
    a = x.abs().max()
    if not torch.isfinite(x).all():
        return torch.zeros_like(x), torch.tensor(math.nan, dtype=torch.float64)
    if float(a) < TINY:
        return torch.zeros_like(x), torch.tensor(0.0, dtype=torch.float64)
    if fmt == "i8":
        return torch.round(x * 127 / a), (a.float() / 127).double()     # torch.round: ties to even; scale rounded once
    m, e = math.frexp(float(a))                                          # a = m 2^e, 1/2 <= m < 1; 448 = 0.875 * 2^9
    scale = 2.0 ** (e - 9 + (1 if m > 0.875 else 0))
    return round_e4m3(x / scale)[0], torch.tensor(scale, dtype=torch.float64)


class Sequence:
    """A sequence's keys and values of one KV head as the cache holds them: rows [n, D] in float64."""

    def __init__(self, k, v, blk, fmt):
        n = k.shape[0]
        self.n, self.blk = n, blk
        full = n // blk
        self.codes, self.scales, self.rows = {}, {}, {}
        for x, t in (("k", k.double()), ("v", v.double())):
            parts = [quantise(t[c * blk:(c + 1) * blk], fmt) for c in range(full)]
            self.codes[x] = torch.stack([p[0] for p in parts]) if full else torch.zeros(0, blk, D, dtype=torch.float64)
            self.scales[x] = torch.stack([p[1] for p in parts]) if full else torch.zeros(0, dtype=torch.float64)
            whole = (self.codes[x] * self.scales[x][:, None, None]).reshape(-1, D)
            self.rows[x] = torch.cat([whole, t[full * blk:]])
        self.bounds = torch.stack([torch.stack([k[c:c + blk].double().amin(0), k[c:c + blk].double().amax(0)])
                                   for c in range(0, n, blk)]) if n else torch.zeros(0, 2, D, dtype=torch.float64)


def candidates(n, window, n_sink):
    hi = max(0, n - window)
    return min(n_sink, hi), hi


def rotate(q, cos, sin):
    a, b = q[..., : D // 2], q[..., D // 2:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def select(q_rot, bounds, n, blk, window, n_sink, top, shared):
    """q_rot [G, D] float64 (the float32 values), bounds [blocks, 2, D] -> per head (blocks ascending, scores float32)."""
    lo, hi = candidates(n, window, n_sink)
    if hi <= lo:
        first, last = 0, 0
    else:
        first, last = lo // blk, (hi - 1) // blk + 1
    s = torch.maximum(q_rot[:, None] * bounds[None, first:last, 0], q_rot[:, None] * bounds[None, first:last, 1]).sum(-1)
    s = s.sum(0, keepdim=True) if shared else s
    s = s.float() + 0.0
    out = []
    for g in range(s.shape[0]):
        order = sorted(range(last - first), key=lambda c: (-float(s[g, c]), c))[:top]
        order.sort()
        out.append(([first + c for c in order], s[g, order]))
    return out


def tokens_of(blocks, n, blk, window, n_sink):
    lo, hi = candidates(n, window, n_sink)
    return [j for c in blocks for j in range(c * blk, (c + 1) * blk) if lo <= j < hi]


def attend(q, q_rot, k, v, n, positions, window, n_sink, cos_win, sin_win, roundings=2 * (128 + 8)):
    """One head.  k, v [n, D] float64; positions: selected candidates.  -> (out [D], error scale [D]): the second is what
    float32 arithmetic of any order may be off by, see `bound`."""
    lo, hi = candidates(n, window, n_sink)
    far = list(range(lo)) + list(positions)
    near = list(range(hi, n))
    if not far and not near:
        return torch.zeros(D, dtype=torch.float64), torch.zeros(D, dtype=torch.float64)
    delta = torch.tensor([n - 1 - j for j in near], dtype=torch.long)
    turned = rotate(q.expand(len(near), D), cos_win[delta], sin_win[delta]) if near else torch.zeros(0, D, dtype=torch.float64)
    heads = torch.cat([q_rot.expand(len(far), D), turned])
    at = torch.tensor(far + near, dtype=torch.long)
    rows, vals = k[at], v[at]
    logit = (heads * rows).sum(-1) / math.sqrt(D)
    p = torch.softmax(logit, 0)
    return p @ vals, bound(heads, rows, p, vals, roundings)


def bound(heads, rows, p, vals, roundings):
    """float32 with u = 2^-24.  A logit is a sum of 128 products of factors with at most three roundings each (a key turned by its
    window position: two products and a sum, 4 u of both halves; scales: 2 u): off by at most (128 + 8) u sum |q k| / sqrt(128),
    where a turned row's |q k| is at most |q| |k|' with both halves: twice as much covers it.  A weight has that in its
    exponent, and 8 u for the exponential and the rescalings (each exp2 argument of size up to 64: 64 u more); sums of weights
    and of p v over the rows add (rows + 16) u.  Numerator and denominator: twice."""
    u = 2.0 ** -24
    d = (roundings * u * (heads.abs() * rows.abs()).sum(-1) / math.sqrt(D)).max() + 72 * u + (len(p) + 16) * u
    return 2 * d * (p @ vals.abs())
