"""Plain float64 forms of the operators on a cache in 4 bits, on the CPU, written from the definitions in include/a2ats.h: rows
and scales as bytes, the numbers that they stand for, and norms of heads with their rotation."""
import math

import torch

D, GROUP = 128, 32
E2M1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
TINY, HUGE = 2.0 ** -100, 2.0 ** 127


def round_group(x):
    """Rows x [..., 32] (float64) -> (codes 0 .. 15, scale bytes [...])."""
    a = x.abs().amax(-1)
    bad = ~torch.isfinite(x).all(-1) | ~(a < HUGE)
    tiny = ~bad & (a < TINY)
    m, e = torch.frexp(torch.where(bad | tiny, torch.ones_like(a), a))     # a = m 2^e, 1/2 <= m < 1; 6 = 0.75 * 2^3
    e = (e - 3 + (m > 0.75).to(e.dtype)).double()
    y = torch.where((bad | tiny)[..., None], torch.zeros_like(x), x).abs() / torch.exp2(e)[..., None]
    up = torch.searchsorted(E2M1, y.contiguous()).clamp(max=7)
    down = (up - 1).clamp(min=0)
    over, under = E2M1[up] - y, y - E2M1[down]
    code = torch.where((over < under) | ((over == under) & (up % 2 == 0)), up, down)
    code = code + 8 * torch.signbit(x).long()
    code = torch.where((bad | tiny)[..., None], 0, code)
    byte = torch.where(bad, 255, torch.where(tiny, 0, (e + 127).long()))
    return code, byte


def numbers(code, byte):
    """What codes [..., 32] with scale bytes [...] stand for."""
    scale = torch.where(byte == 255, math.nan, torch.where(byte == 0, 0.0, torch.exp2(byte.double() - 127)))
    v = E2M1[code % 8]
    return torch.where(code >= 8, -v, v) * scale[..., None]


def cached(k, v):
    """Keys and values [n, 128] -> (rows [n, 128] uint8, scales [n, 8] uint8, keys, values that they stand for)."""
    out, sc, val = [], [], []
    for t in (k, v):
        code, byte = round_group(t.double().unflatten(-1, (D // GROUP, GROUP)))
        sc.append(byte)
        val.append(numbers(code, byte).flatten(-2))
        out.append(code.flatten(-2))
    rows = torch.zeros(k.shape[0], D, dtype=torch.long)
    for d in range(D):
        rows[:, d // 2] |= out[0][:, d] << (4 * (d % 2))
        g, n = d // GROUP, d % GROUP // 2
        rows[:, 64 + 4 * n + g] |= out[1][:, d] << (4 * (d % 2))
    return rows.to(torch.uint8), torch.cat(sc, -1).to(torch.uint8), val[0], val[1]


def bounds(k, blk):
    n = k.shape[0]
    return torch.stack([torch.stack([k[c:c + blk].double().amin(0), k[c:c + blk].double().amax(0)])
                        for c in range(0, n, blk)]) if n else torch.zeros(0, 2, D, dtype=torch.float64)


def norm(x, w, eps):
    """x [..., 128] float64."""
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    return y if w is None else y * w.double()


# Roundings to float32 (2^-24 each) of a normalised element: 13 in the sum of squares (7 additions of a lane and a square's, 4 over the
# lanes, the mean, eps), of which the root halves the effect; the reciprocal root, two steps (2 to 4 roundings); two
# products.  A rotated one: its two products and sum with the table's entries as they are.
NORM_ROUNDINGS = 13 / 2 + 4 + 2
ROTATED_ROUNDINGS = NORM_ROUNDINGS + 3


def half_step(x, dtype):
    """Half a step of the output's type at x (and the least number's)."""
    f = torch.finfo(dtype)
    return f.eps / 2 * x.abs() + f.tiny * f.eps
