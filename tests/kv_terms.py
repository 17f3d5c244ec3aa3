"""Attention over a cache in 8 bits where the low terms of an operand decide: the kernels split queries, turned keys and weights
into a few terms of 8 to 11 bits each, and random data does not show whether the last of them is there.  Inputs, float64 results
and what float32 arithmetic may be off by; `cut` leaves a low term out of the float64 form, to see that it would show."""
import math

import torch

from tests import kv_blocks_ref as R

D, B, HKV, N, BLK, ROWS = 128, 6, 2, 64, 16, 12
U = 2.0 ** -24


class Terms:
    """`what`: "far" - every head attends 12 selected rows; keys have four elements that are not zero, never element 0, and the
    query is 1 in element 0 and about 2^-12 elsewhere, so that what counts are the low bits of its range;
    "window" - the last 12 rows, turned by their distance; keys with four elements, normal queries."""

    def __init__(self, what, fmt, G, shared, seed):
        g = torch.Generator().manual_seed(seed)
        self.what, self.fmt, self.G, self.shared, self.heads = what, fmt, G, shared, HKV * G
        self.window = ROWS if what == "window" else 0
        self.k, self.v = self.codes(g), self.codes(g)
        keep = torch.rand(B, HKV, N, D - 1, generator=g).argsort(-1).argsort(-1) < 4
        self.k[..., 1:] *= keep
        self.k[..., 0] = 0
        spread = 700.0 if what == "far" else 0.16
        self.k_scale = spread * (0.8 + 0.4 * torch.rand(B, HKV, N // BLK, generator=g))
        self.v_scale = 0.01 * (0.8 + 0.4 * torch.rand(B, HKV, N // BLK, generator=g))
        self.q = torch.randn(B, self.heads, D, generator=g)
        self.q_rot = 2.0 ** -12 * torch.randn(B, self.heads, D, generator=g)
        self.q_rot[..., 0] = 1.0
        n_sel = 0 if self.window else ROWS
        H = HKV if shared else self.heads
        self.sel = [[torch.randperm(N, generator=g)[:n_sel].tolist() for _ in range(H)] for _ in range(B)]

    def codes(self, g):
        shape = (B, HKV, N, D)
        if self.fmt == "i8":
            return torch.randint(-127, 128, shape, generator=g).float()
        return (100 * torch.randn(shape, generator=g)).clamp(-448, 448).to(torch.float8_e4m3fn).float()

    def want(self, b, h, cos_win, sin_win, cut=None):
        """-> (out [D], tolerance [D]) of float32 arithmetic."""
        kv = h // self.G
        rows = torch.tensor(list(range(N - ROWS, N)) if self.window else self.sel[b][kv if self.shared else h])
        ks, vs = self.k_scale[b, kv][rows // BLK].double(), self.v_scale[b, kv][rows // BLK].double()
        k, v = self.k[b, kv][rows].double(), self.v[b, kv][rows].double()
        q = (self.q if self.window else self.q_rot)[b, h].double()
        if cut == "query":      # one float16 term
            step = 2.0 ** (torch.floor(torch.log2(q.abs())) - 10)
            q = torch.round(q / step) * step
        if cut == "digit":      # the last of four digits to the base 256
            q = torch.round(q * 2.0 ** 22) / 2.0 ** 22
        if self.window:
            cos, sin = cos_win[N - 1 - rows], sin_win[N - 1 - rows]
            k1, k2 = k[:, : D // 2], k[:, D // 2:]
            size = torch.cat([k1.abs() * cos.abs() + k2.abs() * sin.abs(), k2.abs() * cos.abs() + k1.abs() * sin.abs()], -1)
            k = torch.cat([k1 * cos + k2 * sin, k2 * cos - k1 * sin], -1)       # q R . k = q . (k R^-1)
            if cut == "key":    # one float16 term
                k = k.half().double()
        else:
            size = k.abs()
        logit = k @ q * ks / math.sqrt(D)
        p = torch.softmax(logit, 0)
        out = (p * vs) @ v
        # A logit's roundings, in steps of u = 2^-24 of sum |q| |k|: the query times log2 e / sqrt(128), and that constant (2); a turned
        # key, two products and a sum (3); operands in two float16 terms, to the nearest each: 2^-23 (2 for the key, 2 for the query);
        # the sum of at most 8 elements' products of two terms, exact themselves, each addition of a matrix instruction truncated (32);
        # the sum over the query's terms (3); the scale (1): 45 < 48.  Elements far below the query's largest, 2^(e - 1) <= |q| log2 e / sqrt(128):
        # off by 2^-30 of 2^e (digits; float16 terms: 2^-33).  Terms of a turned key: not below 2^-25.
        size_q = q.abs()
        d = (48 * U * (size @ size_q) * ks / math.sqrt(D)).max()
        low = 2.0 ** -29 * float(q.abs().max()) * k.abs().sum(-1) + (2.0 ** -25 * float(q.abs().sum()) if self.window else 0.0)
        d = d + (low * ks / math.sqrt(D)).max()
        # A weight: the difference to the maximum (its size, times log2 e, u), the exponential (2 u), times v_scale (u); the sums of weights
        # and of three terms times values, 2 u for each of the rows and terms, twice as there are waves to be joined (8 u): 12 u + 6 rows u.
        d = d + (3 * float(logit.abs().max()) + 12 + 6 * len(rows)) * U
        return out, 2 * d * (p * vs) @ v.abs() + U * out.abs()

    def differs(self, cut, cos_win, sin_win):
        """Whether leaving `cut` out is seen in some output."""
        for b in range(B):
            for h in range(self.heads):
                out, tol = self.want(b, h, cos_win, sin_win)
                if ((self.want(b, h, cos_win, sin_win, cut)[0] - out).abs() > 2 * tol).any():
                    return True
        return False


def tables(window):
    """cos / sin of the window's distances as float32 numbers, in float64."""
    inv = torch.exp(-torch.arange(D // 2, dtype=torch.float64) / (D // 2) * math.log(500000.0))
    a = torch.arange(max(window, 1), dtype=torch.float64)[:, None] * inv
    return a.cos().float(), a.sin().float()


ALL = [(what, fmt, G, shared) for what in ("far", "window") for fmt in ("i8", "e4m3") for G, shared in
       ((1, False), (3, True), (4, False), (6, True), (8, True))]
assert R.D == D
