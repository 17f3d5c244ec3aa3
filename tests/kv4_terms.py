"""Attention over a cache in 4 bits where the low terms of an operand decide: large logits that are close to each other, of keys with one
element that is not zero.  Inputs, float64 results and what float32 arithmetic may be off by; `cut` leaves a low term out of
the float64 form, to see that it would show (random data does not show it)."""
import math

import torch

D, B, HKV, N, ROWS = 128, 4, 2, 64, 12
U = 2.0 ** -24
ALL = [(what, G, shared) for what in ("far", "window") for G, shared in ((1, False), (4, False), (3, True), (4, True), (6, True), (8, True))]


class Terms:
    """`what`: "far" - 12 selected rows, each with a 6 in one of four places; "window" - the last 12 rows, each with a 6
    in one of four elements that their distances turn a little."""

    def __init__(self, what, G, shared, seed):
        g = torch.Generator().manual_seed(seed)
        self.what, self.G, self.shared, self.heads = what, G, shared, HKV * G
        self.window = ROWS if what == "window" else 0
        self.k, self.v = torch.zeros(B, HKV, N, D), torch.randint(-4, 5, (B, HKV, N, D), generator=g).float()
        self.v[..., ::32] = 6                              # (scales of 1)
        places = torch.tensor([18, 20, 22, 24] if self.window else [3, 40, 70, 100])
        at = places[torch.randint(0, len(places), (B, HKV, N), generator=g)]
        self.k.scatter_(-1, at[..., None], 6.0)
        self.q = torch.zeros(B, self.heads, D)
        size = 60 + 40 * torch.rand(B, self.heads, 1, generator=g)
        self.q[..., places] = size * (1 + 0.01 * torch.randn(B, self.heads, len(places), generator=g))
        H = HKV if shared else self.heads
        self.sel = [[[] if self.window else torch.randperm(N, generator=g)[:ROWS].tolist() for _ in range(H)] for _ in range(B)]

    def want(self, b, h, cos_win, sin_win, cut=None):
        """-> (out [D], tolerance [D]) of float32 arithmetic."""
        kv = h // self.G
        rows = torch.tensor(list(range(N - ROWS, N)) if self.window else self.sel[b][kv if self.shared else h])
        k, v, q = self.k[b, kv][rows].double(), self.v[b, kv][rows].double(), self.q[b, h].double()
        if cut == "query":      # 16 bits
            step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -100))) - 15)
            q = torch.trunc(q / step) * step
        if self.window:
            cos, sin = cos_win[N - 1 - rows], sin_win[N - 1 - rows]
            k1, k2 = k[:, : D // 2], k[:, D // 2:]
            k = torch.cat([k1 * cos + k2 * sin, k2 * cos - k1 * sin], -1)       # q R . k = q . (k R^-1)
            if cut == "key":    # one float16 term
                k = k.half().double()
        logit = k @ q / math.sqrt(D)
        p = torch.softmax(logit, 0)
        # A logit's roundings, in steps of u = 2^-24 of it: the query times log2 e / sqrt(128), and that constant (2); a turned key's product
        # (1); float16 terms, to the nearest each (2 for the key, 2 for the query); the products of two terms of the key, added by the
        # matrix cores and truncated (2 x 2); the sum over the query's terms (3): 14 < 16.  (Far keys: exact but for the first and the last.)
        d = 16 * U * float(logit.abs().max())
        # A weight: the difference to the maximum (its size u), the exponential (2 u); the sums of weights and of three terms times
        # values, 2 u for each of the rows and terms, twice as there are waves to be joined (8 u): 12 u + 6 rows u.
        d = d + (3 * float(logit.abs().max()) + 12 + 6 * len(rows)) * U
        out = p @ v
        return out, 2 * d * (p @ v.abs()) + U * out.abs()

    def differs(self, cut, cos_win, sin_win):
        """Whether leaving `cut` out is seen in some output."""
        for b in range(B):
            for h in range(self.heads):
                out, tol = self.want(b, h, cos_win, sin_win)
                if ((self.want(b, h, cos_win, sin_win, cut)[0] - out).abs() > 2 * tol).any():
                    return True
        return False


def tables(window):
    """cos / sin of the window's distances as float32 numbers."""
    inv = torch.exp(-torch.arange(D // 2, dtype=torch.float64) / (D // 2) * math.log(500000.0))
    a = torch.arange(max(window, 1), dtype=torch.float64)[:, None] * inv
    return a.cos().float(), a.sin().float()
