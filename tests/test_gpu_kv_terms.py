"""Attention over a cache in 8 bits: the terms that its operands are split into are all there, for every number of heads that
attend the same rows (tests/kv_terms.py)."""
import pytest
import torch

from paper_2502_12665_amd import binding as B
from tests import kv_terms as K

pytestmark = pytest.mark.gpu
D = 128
CODES = {"i8": torch.int8, "e4m3": torch.float8_e4m3fn}


def attend(dims, cache, q, q_rot, sel, size, shared, window, cos_win, sin_win):
    """sel [B][H] lists of the same number, or of none."""
    n_sel = max(1, len(sel[0][0]))
    idx = torch.tensor([[row if row else [-1] for row in rows] for rows in sel], dtype=torch.int32).cuda()
    cnt = torch.full(idx.shape[:2], len(sel[0][0]), dtype=torch.int32).cuda()
    ws = torch.empty(max(16, B.workspace_bytes(dims, B.OP_ATTN_KV8, n_sel * size, window)), dtype=torch.uint8, device="cuda")
    out = torch.full_like(q, 3.0, device="cuda")
    B.sparse_attn_kv8(dims, cache, q.cuda(), q_rot.cuda(), idx, cnt, n_sel, size, shared, window, 0, cos_win.contiguous().cuda(),
                      sin_win.contiguous().cuda(), None, out, ws)
    torch.cuda.synchronize()
    return out.cpu()


def filled(dims, dtype, fmt, k, v, k_scale, v_scale, blk):
    cache = B.KvBlocks.empty(dims, blk, dtype, CODES[fmt], False)
    for x, codes, scale in (("k", k, k_scale), ("v", v, v_scale)):
        getattr(cache, x).copy_(codes.to(CODES[fmt]))
        getattr(cache, x + "_scale").copy_(scale)
    return cache


@pytest.mark.parametrize("what, fmt, G, shared", K.ALL)
def test_low_terms_of_queries_and_keys(what, fmt, G, shared):
    t = K.Terms(what, fmt, G, shared, seed=G)
    dims = B.make_dims(K.B, t.heads, K.HKV, D, 16, K.N, K.N)
    cache = filled(dims, torch.float32, fmt, t.k, t.v, t.k_scale, t.v_scale, K.BLK)
    cos, sin = K.tables(t.window)
    got = attend(dims, cache, t.q, t.q_rot, t.sel, 1, shared, t.window, cos, sin)
    for b in range(K.B):
        for h in range(t.heads):
            want, tol = t.want(b, h, cos.double(), sin.double())
            err = (got[b, h].double() - want).abs()
            assert (err <= tol).all(), (b, h, float((err / tol).max()), float(err.max()))


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("G, shared", [(1, False), (4, False), (3, True), (4, True), (5, True), (6, True), (7, True), (8, True)])
@pytest.mark.parametrize("window", [0, 1])
def test_weights_have_24_bits(fmt, G, shared, window):
    """A query of zeros and one row: the weight is that row's v_scale, any float32.  Its three terms hold all of it, their products with a
    code are exact, and at most three additions follow (a truncated one is off by 2 u), and a division by 1: 7 u < 8 u.  Weights of
    16 bits are off by up to 2^-16 = 256 u."""
    batch, n, blk, Hkv = 24, 16, 16, 2
    heads = Hkv * G
    g = torch.Generator().manual_seed(G + window)
    v = torch.randint(-127, 128, (batch, Hkv, n, D), generator=g).float() if fmt == "i8" else \
        (100 * torch.randn(batch, Hkv, n, D, generator=g)).clamp(-448, 448).to(torch.float8_e4m3fn).float()
    v_scale = torch.rand(batch, Hkv, 1, generator=g) + 0.01
    dims = B.make_dims(batch, heads, Hkv, D, 16, n, n)
    cache = filled(dims, torch.float32, fmt, v, v, v_scale, v_scale, blk)
    zero = torch.zeros(batch, heads, D)
    H = Hkv if shared else heads
    pick = torch.randint(0, n - 1, (batch, H, 1), generator=g)
    sel = [[[] for _ in range(H)] for _ in range(batch)] if window else pick.tolist()
    cos, sin = K.tables(window)
    got = attend(dims, cache, zero, zero, sel, 1, shared, window, cos, sin)
    for b in range(batch):
        for h in range(heads):
            row = n - 1 if window else sel[b][h // G if shared else h][0]
            want = v[b, h // G, row].double() * v_scale[b, h // G, 0].double()
            err = (got[b, h].double() - want).abs()
            assert (err <= 8 * 2.0 ** -24 * want.abs()).all(), (b, h, float((err / want.abs().clamp(min=1e-30)).max() * 2 ** 24))


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("G, shared", [(4, False), (4, True), (5, True), (8, True)])
@pytest.mark.parametrize("window", [0, 1])
def test_weights_next_to_a_border_of_bfloat16(fmt, G, shared, window):
    """Outputs 2^-18 above and below the middle of two bfloat16 numbers (8 u = 2^-21 is what they may be off by before their rounding):
    a weight cut to 16 bits rounds the upper one down."""
    batch, n, blk, Hkv = 2, 16, 16, 1
    dims = B.make_dims(batch, G, Hkv, D, 16, n, n)
    v = torch.ones(batch, Hkv, n, D)
    v[..., ::2] = -1
    scale = torch.tensor([1 + 2.0 ** -8 + 2.0 ** -18, 1 + 2.0 ** -8 - 2.0 ** -18]).reshape(2, 1, 1)
    cache = filled(dims, torch.bfloat16, fmt, v, v, scale, scale, blk)
    zero = torch.zeros(batch, G, D)
    H = Hkv if shared else G
    sel = [[[] if window else [3]] * H] * batch
    cos, sin = K.tables(window)
    got = attend(dims, cache, zero.bfloat16(), zero, sel, 1, shared, window, cos, sin).double()
    assert (got[0].abs() == 1 + 2.0 ** -7).all() and (got[1].abs() == 1).all()
    assert (torch.sign(got) == torch.sign(v[:, :, 3])).all()


@pytest.mark.parametrize("G, shared", [(4, False), (4, True), (7, True)])
@pytest.mark.parametrize("fmt, dtype", [("i8", torch.float32), ("i8", torch.bfloat16), ("e4m3", torch.float32)])
def test_queries_of_zeros_and_tiny_ones(fmt, dtype, G, shared):
    """Queries of 2^-99 (and of zeros: all rows alike) over keys whose scales make ordinary logits of them."""
    batch, n, blk, Hkv, rows = 3, 32, 16, 1, 8
    g = torch.Generator().manual_seed(5)
    dims = B.make_dims(batch, G, Hkv, D, 16, n, n)
    k = torch.zeros(batch, Hkv, n, D)
    k[..., 3] = torch.randint(-100, 101, (batch, Hkv, n), generator=g).float()
    k[..., 80] = torch.randint(-100, 101, (batch, Hkv, n), generator=g).float()
    if fmt == "e4m3":
        k = k.to(torch.float8_e4m3fn).float()
    v = torch.randint(-8, 9, (batch, Hkv, n, D), generator=g).float()
    k_scale = torch.full((batch, Hkv, n // blk), 2.0 ** 95)
    v_scale = torch.full((batch, Hkv, n // blk), 0.25)
    cache = filled(dims, dtype, fmt, k, v, k_scale, v_scale, blk)
    q_rot = torch.zeros(batch, G, D)
    for b, s in enumerate((0.0, 2.0 ** -97, 2.0 ** -99)):
        q_rot[b, :, 3], q_rot[b, :, 80] = s, -0.75 * s
    H = Hkv if shared else G
    sel = [[torch.randperm(n, generator=g)[:rows].tolist() for _ in range(H)] for _ in range(batch)]
    cos, sin = K.tables(0)
    got = attend(dims, cache, q_rot.to(dtype), q_rot, sel, 1, shared, 0, cos, sin)
    for b in range(batch):
        for h in range(G):
            at = sel[b][0 if shared else h]
            kk, vv = k[b, 0, at].double() * 2.0 ** 95, v[b, 0, at].double() * 0.25
            logit = kk @ q_rot[b, h].double() / D ** 0.5
            p = logit.softmax(0)
            # 16 u of the products (two elements: fewer roundings than tests/kv_terms.py counts), 12 u and 6 u a row for the weights
            d = 16 * K.U * float((kk.abs() @ q_rot[b, h].double().abs()).max()) / D ** 0.5 + (3 * float(logit.abs().max()) + 12 + 6 * rows) * K.U
            half = 2.0 ** -8 if dtype == torch.bfloat16 else K.U
            want = p @ vv
            assert ((got[b, h].double() - want).abs() <= 2 * d * (p @ vv.abs()) * (1 + half) + half * want.abs()).all(), (b, h)
