"""Host side of the operators on a cache in 4 bits, and of the norms: what they refuse before anything is launched, their
workspaces, what the binding checks, and the plain forms that the GPU tests compare with.  No GPU."""
import ctypes

import pytest
import torch

from tests import kv4_ref as R
from tests import kv4_terms as K


@pytest.fixture(scope="module")
def B():
    from paper_2502_12665_amd import binding as b
    b.lib()
    return b


ONE = 16     # non-NULL, aligned, never dereferenced: validation fails first (or there is no batch)


def cache(B, **kw):
    f = dict(rows=ONE, scales=ONE, bounds=ONE, page_table=None, page_size=0, block=32, kv_dtype=1)
    f.update(kw)
    return B.Kv4Struct(*[f[x[0]] for x in B.Kv4Struct._fields_])


def dims(B, batch=0, heads=8, kv_heads=2, n=100, stride=128, d=128):
    """batch 0: a call that passes every check enqueues nothing and needs no GPU."""
    return B.make_dims(batch, heads, kv_heads, d, 16, n, stride)


BAD_CACHES = [(dict(block=0), -1), (dict(block=8), -1), (dict(block=48), -1), (dict(block=256), -2), (dict(kv_dtype=2), -1),
              (dict(page_table=ONE, page_size=16), -1), (dict(page_table=ONE, page_size=96), -1), (dict(page_table=ONE, page_size=0), -1),
              (dict(rows=None), -1), (dict(rows=8), -1), (dict(scales=None), -1), (dict(scales=4), -1), (dict(bounds=8), -1)]
BAD_DIMS = [(dict(kv_heads=3), -1), (dict(d=64), -2), (dict(heads=32, kv_heads=2), -2), (dict(stride=99), -1),
            (dict(n=1 << 21, stride=1 << 21), -2), (dict(batch=-1), -1)]


def append(B, d=None, c=None, k=ONE, v=ONE, n_new=1):
    return B.lib().a2ats_kv4_append(ctypes.byref(d or dims(B)), ctypes.byref(c or cache(B)), k, v, n_new, None, None, None)


def read(B, d=None, c=None, n_rows=1, k=ONE, v=ONE, dtype=0):
    return B.lib().a2ats_kv4_read(ctypes.byref(d or dims(B)), ctypes.byref(c or cache(B)), n_rows, None, None, k, v, dtype, None)


def attn(B, d=None, c=None, q=ONE, q_rot=ONE, idx=ONE, cnt=ONE, n_sel=4, size=1, window=8, sink=0, cos=ONE, sin=ONE, out=ONE, ws=None,
         ws_bytes=0, shared=0):
    return B.lib().a2ats_sparse_attn_kv4(ctypes.byref(d or dims(B)), ctypes.byref(c or cache(B)), q, q_rot, idx, cnt, n_sel, size, shared,
                                         window, sink, cos, sin, None, out, ws, ws_bytes, None)


def norm(B, d=None, q=ONE, qs=1024, k=ONE, ks=256, dtype=1, n_new=1, qw=ONE, kw=ONE, eps=1e-6, cos=ONE, sin=ONE, n_pos=100, qn=ONE,
         kn=ONE, qp=ONE, kp=ONE):
    return B.lib().a2ats_qk_norm_rope(ctypes.byref(d or dims(B)), q, qs, k, ks, dtype, n_new, qw, kw, eps, cos, sin, n_pos, None, None,
                                      qn, kn, qp, kp, None)


def test_what_is_allowed_passes_every_check(B):
    for c in (cache(B), cache(B, kv_dtype=0, bounds=None), cache(B, page_table=ONE, page_size=32), cache(B, scales=8)):
        assert append(B, c=c) == 0 and append(B, c=c, n_new=0) == 0 and append(B, c=c, n_new=100) == 0
        assert read(B, c=c) == 0 and read(B, c=c, k=None) == 0 and read(B, c=c, v=None, dtype=1) == 0 and read(B, c=c, n_rows=100) == 0
        assert attn(B, c=c) == 0 and attn(B, c=c, size=32) == 0 and attn(B, c=c, n_sel=0, idx=None, window=0, cos=None, sin=None) == 0
    assert append(B, d=dims(B, stride=101), c=cache(B, page_table=ONE, page_size=64)) == 0   # (pages: any stride)
    assert norm(B) == 0 and norm(B, qw=None, kw=None) == 0 and norm(B, qs=1544, ks=1544) == 0 and norm(B, n_new=100, dtype=0) == 0
    assert norm(B, k=None, kn=None, kp=None, ks=0) == 0 and norm(B, q=None, qn=None, qp=None, qs=0) == 0
    assert norm(B, qp=None, kp=None, cos=None, sin=None, n_pos=0) == 0 and norm(B, qn=None, kp=None) == 0
    assert norm(B, eps=1.0) == 0 and norm(B, eps=2.0 ** -126) == 0


def test_caches_that_are_refused(B):
    for kw, rc in BAD_CACHES:
        for call in (append, read, attn):
            assert call(B, c=cache(B, **kw)) == rc, (kw, call)
    for kw, rc in BAD_DIMS + [(dict(stride=112), -1)]:      # (112: no multiple of the block)
        for call in (append, read, attn):
            assert call(B, d=dims(B, **kw)) == rc, (kw, call)
    for kw, rc in BAD_DIMS:
        assert norm(B, d=dims(B, **kw)) == rc, kw
    L = B.lib()
    assert L.a2ats_kv4_append(ctypes.byref(dims(B)), None, ONE, ONE, 1, None, None, None) == -1
    assert L.a2ats_kv4_read(None, ctypes.byref(cache(B)), 1, None, None, ONE, ONE, 0, None) == -1


def test_arguments_that_are_refused(B):
    for kw in (dict(k=None), dict(v=None), dict(k=8), dict(v=8), dict(n_new=-1), dict(n_new=101)):
        assert append(B, **kw) == -1, kw
    for kw in (dict(k=None, v=None), dict(k=8), dict(v=8), dict(n_rows=-1), dict(n_rows=101), dict(dtype=2), dict(dtype=-1)):
        assert read(B, **kw) == -1, kw
    for kw in (dict(q=None), dict(q=8), dict(q_rot=None), dict(q_rot=8), dict(idx=None), dict(cnt=None), dict(n_sel=-1), dict(window=-1),
               dict(sink=-1), dict(cos=None), dict(sin=None), dict(cos=8), dict(out=None), dict(size=16), dict(size=0), dict(size=64)):
        assert attn(B, **kw) == -1, kw
    assert attn(B, n_sel=4097) == -2
    for kw in (dict(q=None, k=None), dict(q=None), dict(k=None), dict(qs=1016), dict(ks=248), dict(qs=1028), dict(ks=260), dict(dtype=2), dict(n_new=-1), dict(n_new=101),
               dict(eps=0.0), dict(eps=-1.0), dict(eps=2.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(cos=None), dict(sin=None),
               dict(n_pos=99), dict(qn=None, qp=None), dict(kn=None, kp=None), dict(q=8), dict(k=8), dict(qw=8), dict(kw=8), dict(cos=8),
               dict(sin=8), dict(qn=8), dict(kn=8), dict(qp=8), dict(kp=8)):
        assert norm(B, **kw) == -1, kw


def test_workspaces(B):
    long = dims(B, batch=1, n=100000, stride=100000 // 32 * 32 + 32)
    need = B.workspace_bytes(long, B.OP_ATTN_KV4, 2048, 64)
    assert need > 0 and attn(B, d=long, n_sel=2048, window=64) == -3 and attn(B, d=long, n_sel=2048, window=64, ws=ONE, ws_bytes=64) == -3
    assert attn(B, d=long, n_sel=2048, window=64, ws=8, ws_bytes=need) == -3
    for bad in ((-1, 0), (0, -1)):
        with pytest.raises(B.A2atsError):
            B.workspace_bytes(dims(B, batch=1), B.OP_ATTN_KV4, *bad)
    last = 0
    for n_sel in (0, 1, 64, 500, 1000, 4096, 4096 * 128):
        w = B.workspace_bytes(dims(B, batch=1, n=1 << 20, stride=1 << 20), B.OP_ATTN_KV4, n_sel, 64)
        assert w >= last
        last = w


def test_calls_of_nothing(B):
    one = dims(B, batch=1)
    assert append(B, d=one, k=None, v=None, n_new=0) == 0 and read(B, d=one, k=None, v=None, n_rows=0) == 0
    assert norm(B, d=one, q=None, k=None, n_new=0) == 0


def test_grids_that_are_too_large_are_refused(B):
    """Launches of 2^32 threads or more."""
    many = dims(B, batch=1 << 20, heads=8, kv_heads=8)
    assert append(B, d=many) == -2 and attn(B, d=dims(B, batch=1 << 21, heads=8, kv_heads=8)) == -2
    assert read(B, d=dims(B, batch=1 << 21, heads=8, kv_heads=8)) == -2
    assert norm(B, d=dims(B, batch=1 << 20), n_new=64) == -2
    big = dims(B, batch=1 << 18, heads=64, kv_heads=64, n=1 << 20, stride=1 << 20)
    assert append(B, d=big, n_new=1 << 20) == -2 and read(B, d=big, n_rows=1 << 20) == -2
    assert norm(B, d=big, qs=8192, ks=8192, n_new=1 << 20, n_pos=1 << 20) == -2


def test_binding_refuses_what_does_not_fit(B):
    d = dims(B, batch=2)
    bf, f32 = torch.bfloat16, torch.float32
    c = B.Kv4Cache.empty(d, 32, bf, device="cpu")
    assert tuple(c.rows.shape) == (2, 2, 128, 128) and tuple(c.scales.shape) == (2, 2, 128, 8) and tuple(c.bounds.shape) == (2, 2, 4, 2, 128)
    assert c.blocks.bounds is c.bounds and c.blocks.k is None and B.Kv4Cache.empty(d, 64, f32, False, device="cpu").blocks is None
    table = torch.zeros(2, 4, dtype=torch.int32)
    p = B.Kv4Cache.empty(d, 32, bf, True, table, 32, 9, device="cpu")
    assert tuple(p.rows.shape) == (9, 2, 32, 128) and tuple(p.bounds.shape) == (9, 2, 1, 2, 128)
    for err, a in ((TypeError, (d, 32, bf, c.rows.to(torch.int8), c.scales)), (ValueError, (d, 32, bf, c.rows[:, :, :64], c.scales)),
                   (ValueError, (d, 32, bf, c.rows, c.scales[..., :4])), (ValueError, (d, 24, bf, c.rows, c.scales)),
                   (TypeError, (d, 32, torch.float16, c.rows, c.scales)), (TypeError, (d, 32, f32, c.rows, c.scales, c.bounds)),
                   (ValueError, (d, 64, bf, c.rows, c.scales, c.bounds)), (ValueError, (dims(B, batch=2, stride=120), 16, bf, c.rows, c.scales)),
                   (ValueError, (d, 32, bf, p.rows, p.scales, p.bounds, table, 16)),
                   (TypeError, (d, 32, bf, p.rows, p.scales, p.bounds, table.long(), 32)),
                   (ValueError, (d, 32, bf, p.rows, p.scales, p.bounds[:8], table, 32)),
                   (ValueError, (d, 32, bf, c.rows.transpose(0, 1).contiguous().transpose(0, 1), c.scales))):
        with pytest.raises(err):
            B.Kv4Cache(*a)
    x = torch.zeros(2, 2, 1, 128, dtype=bf)
    for call in (lambda: B.kv4_append(d, c, x, x, 1), lambda: B.kv4_read(d, c, 1, None, None, x, x), lambda: B.kv4_read(d, c, 1, None, None, None, None),
                 lambda: B.kv4_append(dims(B, batch=3), c, x, x, 1),
                 lambda: B.qk_norm_rope(d, None, None, 1, None, None, 1e-6, None, None),
                 lambda: B.qk_norm_rope(d, torch.zeros(2, 1, 1024), None, 1, None, None, 1e-6, None, None)):   # (host memory)
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        B.BlockDecodeState(d, B.Kv4Cache.empty(d, 64, f32, False, device="cpu"), 1, 8, 0, torch.ones(64, dtype=torch.float64), 4)


def test_layouts_of_projections(B):
    """Strides that the norms are given: slices of one projection, tensors of their own, heads as an axis; others are refused."""
    d = dims(B, batch=3)
    qkv = torch.zeros(3, 5, 1024 + 512)
    assert B._projected(d, qkv[..., :1024], "q", 8, 5) == (qkv.data_ptr(), 1536)
    assert B._projected(d, qkv[..., 1024:1280], "k", 2, 5) == (qkv.data_ptr() + 4096, 1536)
    assert B._projected(d, qkv[..., :1024].unflatten(-1, (8, 128)), "q", 8, 5)[1] == 1536
    assert B._projected(d, torch.zeros(3, 1, 1024), "q", 8, 1)[1] == 1024 and B._projected(d, qkv[:, :1, :1024], "q", 8, 1)[1] == 5 * 1536
    assert B._projected(dims(B, batch=1), qkv[:1, 2:4, :1024], "q", 8, 2)[1] == 1536
    for bad, n in ((qkv[:, :4, :1024], 4), (qkv[..., :512], 5), (qkv[..., ::2][..., :768], 5), (torch.zeros(5, 3, 1024).transpose(0, 1), 5),
                   (torch.zeros(3, 5, 128, 8).transpose(2, 3), 5), (qkv[..., :1024], 4)):
        with pytest.raises(ValueError):
            B._projected(d, bad, "q", 8, n)


def test_the_plain_forms_themselves():
    """Rounding by hand; packing against the order that the header states, byte by byte; norms."""
    x = torch.zeros(1, 32, dtype=torch.float64)
    x[0, :16] = torch.tensor([6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -0.75, -5, 0.2500001, 0.7499999, 4.9999, -0.0, 5.0001])
    code, byte = R.round_group(x)
    assert byte.tolist() == [127] and code[0, :16].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 8, 10, 14, 1, 1, 6, 8, 7]
    for a, want in ((6.0, 127), (6.0000001, 128), (3.0, 126), (2.0 ** -100, 127 - 102), (2.0 ** -101, 0), (2.0 ** 127, 255), (1.9 * 2.0 ** 126, 252),
                    (float("inf"), 255), (float("nan"), 255)):
        x = torch.zeros(1, 32, dtype=torch.float64)
        x[0, 3] = a
        assert R.round_group(x)[1].item() == want, a
    g = torch.Generator().manual_seed(1)
    k, v = torch.randn(7, 128, generator=g).bfloat16(), torch.randn(7, 128, generator=g).bfloat16()
    rows, scales, kk, vv = R.cached(k, v)
    for d in range(128):
        for t, val, byte, sc in ((kk, k, d // 2, d // 32), (vv, v, 64 + 4 * (d % 32 // 2) + d // 32, 4 + d // 32)):
            code = (rows[:, byte].long() >> (4 * (d % 2))) & 15
            want = R.E2M1[code % 8] * torch.where(code >= 8, -1.0, 1.0) * torch.exp2(scales[:, sc].double() - 127)
            assert torch.equal(t[:, d], want)
    step = torch.exp2(scales[:, :4].double() - 127).repeat_interleave(32, -1)
    assert ((kk - k.double()).abs() <= step).all() and (kk.abs() <= 6 * step).all()
    x = torch.randn(3, 128, generator=g).double()
    assert torch.allclose(R.norm(x, None, 1e-6).square().mean(-1), torch.ones(3, dtype=torch.float64), atol=1e-4)


@pytest.mark.parametrize("what, G, shared", K.ALL)
def test_a_low_term_that_is_left_out_would_show(what, G, shared):
    t = K.Terms(what, G, shared, seed=G)
    cos, sin = (x.double() for x in K.tables(t.window))
    for cut in ("query",) + (("key",) if what == "window" else ()):
        assert t.differs(cut, cos, sin), cut
    for x in (t.k, t.v):                                    # held exactly in 4 bits
        _, _, a, _ = R.cached(x[0, 0], x[0, 0])
        assert torch.equal(a, x[0, 0].double())
