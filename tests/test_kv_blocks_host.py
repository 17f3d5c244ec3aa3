"""Host side of the operators on a cache cut into blocks: what they refuse before anything is launched, their workspaces, and
what the binding checks.  No GPU."""
import ctypes

import pytest
import torch

from tests import kv_blocks_ref as R


@pytest.fixture(scope="module")
def B():
    from paper_2502_12665_amd import binding as b
    b.lib()
    return b


ONE = 16     # non-NULL, aligned, never dereferenced: validation fails first (or there is no batch)


def blocks(B, **kw):
    f = dict(k=ONE, v=ONE, k_scale=ONE, v_scale=ONE, k_tail=ONE, v_tail=ONE, bounds=ONE, page_table=None, page_size=0, block=32,
             format=0, kv_dtype=1)
    f.update(kw)
    return B.KvBlocksStruct(*[f[x[0]] for x in B.KvBlocksStruct._fields_])


def dims(B, batch=0, heads=8, kv_heads=2, n=100, stride=128, d=128):
    """batch 0: a call that passes every check enqueues nothing and needs no GPU."""
    return B.make_dims(batch, heads, kv_heads, d, 16, n, stride)


BAD_BLOCKS = [(dict(block=0), -1), (dict(block=8), -1), (dict(block=48), -1), (dict(block=256), -2), (dict(kv_dtype=2), -1),
              (dict(page_table=ONE, page_size=16), -1), (dict(page_table=ONE, page_size=96), -1), (dict(page_table=ONE, page_size=0), -1)]
BAD_ROWS = [(dict(format=2), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(k_scale=None), -1), (dict(v_scale=None), -1),
            (dict(k_tail=None), -1), (dict(v_tail=None), -1), (dict(k=8), -1), (dict(v=4), -1), (dict(k_tail=8), -1), (dict(v_tail=8), -1),
            (dict(bounds=8), -1)]
BAD_DIMS = [(dict(kv_heads=3), -1), (dict(d=64), -2), (dict(heads=32, kv_heads=2), -2), (dict(stride=99), -1), (dict(stride=112), -1),
            (dict(n=1 << 21, stride=1 << 21), -2), (dict(batch=-1), -1)]


def append(B, d=None, bl=None, k=ONE, v=ONE, n_new=1):
    return B.lib().a2ats_kv8_append(ctypes.byref(d or dims(B)), ctypes.byref(bl or blocks(B)), k, v, n_new, None, None, None)


def bounds(B, d=None, bl=None, k=ONE, n_new=1):
    return B.lib().a2ats_key_bounds(ctypes.byref(d or dims(B)), ctypes.byref(bl or blocks(B)), k, n_new, None, None, None)


def topk(B, d=None, bl=None, q=ONE, cos=ONE, sin=ONE, q_rot=ONE, top=4, window=8, sink=0, idx=ONE, cnt=ONE, tok=None, ntok=None, ws=None,
         ws_bytes=0, shared=0):
    return B.lib().a2ats_block_topk(ctypes.byref(d or dims(B)), ctypes.byref(bl or blocks(B)), q, cos, sin, q_rot, shared, top, window,
                                    sink, None, idx, cnt, None, tok, ntok, ws, ws_bytes, None)


def attn(B, d=None, bl=None, q=ONE, q_rot=ONE, idx=ONE, cnt=ONE, n_sel=4, size=1, window=8, sink=0, cos=ONE, sin=ONE, out=ONE, ws=None,
         ws_bytes=0, shared=0):
    return B.lib().a2ats_sparse_attn_kv8(ctypes.byref(d or dims(B)), ctypes.byref(bl or blocks(B)), q, q_rot, idx, cnt, n_sel, size, shared,
                                         window, sink, cos, sin, None, out, ws, ws_bytes, None)


def test_what_is_allowed_passes_every_check(B):
    for bl in (blocks(B), blocks(B, format=1, kv_dtype=0, bounds=None), blocks(B, page_table=ONE, page_size=32)):
        assert append(B, bl=bl) == 0 and append(B, bl=bl, n_new=0) == 0 and append(B, bl=bl, n_new=100) == 0
        assert attn(B, bl=bl) == 0 and attn(B, bl=bl, size=32) == 0 and attn(B, bl=bl, n_sel=0, idx=None, window=0, cos=None, sin=None) == 0
    only = blocks(B, k=None, v=None, k_scale=None, v_scale=None, k_tail=None, v_tail=None, format=9)
    assert bounds(B, bl=only) == 0 and topk(B, bl=only) == 0 and topk(B, bl=only, top=0, idx=None) == 0
    assert topk(B, tok=ONE, ntok=ONE) == 0
    assert append(B, d=dims(B, stride=101), bl=blocks(B, page_table=ONE, page_size=64)) == 0   # (pages: any stride)


def test_caches_that_are_refused(B):
    for kw, rc in BAD_BLOCKS:
        for call in (append, bounds, topk, attn):
            assert call(B, bl=blocks(B, **kw)) == rc, (kw, call)
    for kw, rc in BAD_ROWS:
        for call in (append, attn):
            assert call(B, bl=blocks(B, **kw)) == rc, (kw, call)
    for call in (bounds, topk):
        assert call(B, bl=blocks(B, bounds=None)) == -1 and call(B, bl=blocks(B, bounds=8)) == -1
    for kw, rc in BAD_DIMS:
        for call in (append, bounds, topk, attn):
            assert call(B, d=dims(B, **kw)) == rc, (kw, call)
    L = B.lib()
    assert L.a2ats_kv8_append(ctypes.byref(dims(B)), None, ONE, ONE, 1, None, None, None) == -1
    assert L.a2ats_kv8_append(None, ctypes.byref(blocks(B)), ONE, ONE, 1, None, None, None) == -1


def test_arguments_that_are_refused(B):
    assert append(B, k=None) == -1 and append(B, v=None) == -1 and append(B, k=8) == -1 and append(B, v=8) == -1
    assert append(B, n_new=-1) == -1 and append(B, n_new=101) == -1 and bounds(B, k=None) == -1 and bounds(B, n_new=101) == -1
    big = dims(B, batch=1 << 18, heads=64, kv_heads=64, n=1 << 20, stride=1 << 20)
    assert append(B, d=big, n_new=1 << 20) == -2
    for kw in (dict(q=None), dict(q=8), dict(cos=None), dict(sin=None), dict(cos=8), dict(q_rot=None), dict(q_rot=8), dict(idx=None),
               dict(cnt=None), dict(top=-1), dict(window=-1), dict(sink=-1), dict(tok=ONE), dict(ntok=ONE)):
        assert topk(B, **kw) == -1, kw
    assert topk(B, top=4097) == -2
    one = dims(B, batch=1)
    need = B.workspace_bytes(one, B.OP_BLOCK_TOPK)
    assert need > 0 and topk(B, d=one) == -3 and topk(B, d=one, ws=8, ws_bytes=need) == -3
    assert topk(B, d=one, ws=ONE, ws_bytes=8 * 4 * 4 - 1) == -3               # 8 heads x 4 blocks of 32
    for kw in (dict(q=None), dict(q=8), dict(q_rot=None), dict(q_rot=8), dict(idx=None), dict(cnt=None), dict(n_sel=-1), dict(window=-1),
               dict(sink=-1), dict(cos=None), dict(sin=None), dict(cos=8), dict(out=None), dict(size=16), dict(size=0), dict(size=64)):
        assert attn(B, **kw) == -1, kw
    assert attn(B, n_sel=4097) == -2
    long = dims(B, batch=1, n=100000, stride=100000 // 32 * 32 + 32)
    need = B.workspace_bytes(long, B.OP_ATTN_KV8, 2048, 64)
    assert need > 0 and attn(B, d=long, n_sel=2048, window=64) == -3 and attn(B, d=long, n_sel=2048, window=64, ws=ONE, ws_bytes=64) == -3


def test_calls_of_nothing(B):
    """No new tokens, or no blocks to select: the empty arrays may have no address."""
    one = dims(B, batch=1)
    assert append(B, d=one, k=None, v=None, n_new=0) == 0 and bounds(B, d=one, k=None, n_new=0) == 0
    assert topk(B, top=0, idx=None, tok=None, ntok=ONE) == 0


def test_grids_that_are_too_large_are_refused(B):
    """Launches of 2^32 threads or more."""
    many = dims(B, batch=1 << 20, heads=8, kv_heads=8)
    assert append(B, d=many) == -2 and topk(B, d=many) == -2
    assert attn(B, d=dims(B, batch=1 << 21, heads=8, kv_heads=8)) == -2


def test_workspaces_cover_their_calls(B):
    """The figure for the smallest blocks and 64 sinks is enough for every block size, kind of selection and fewer sinks: found by
    asking the calls, which refuse what is too small (a batch of one, so that nothing is launched: ws misaligned at the figure)."""
    with pytest.raises(B.A2atsError):
        B.workspace_bytes(dims(B, batch=1), B.OP_ATTN_KV8, -1, 0)
    last = 0
    for n_sel in (0, 1, 64, 500, 1000, 4096, 4096 * 128):
        w = B.workspace_bytes(dims(B, batch=1, n=1 << 20, stride=1 << 20), B.OP_ATTN_KV8, n_sel, 64)
        assert w >= last
        last = w
    assert B.workspace_bytes(dims(B, batch=3, n=1000, stride=1024), B.OP_BLOCK_TOPK) >= 3 * 8 * 63 * 4


def test_binding_refuses_what_does_not_fit(B):
    d = dims(B, batch=2)
    bf, f32 = torch.bfloat16, torch.float32
    c = B.KvBlocks.empty(d, 32, bf, device="cpu")
    assert c.format == B.I8 and tuple(c.k.shape) == (2, 2, 128, 128) and tuple(c.bounds.shape) == (2, 2, 4, 2, 128)
    assert B.KvBlocks.empty(d, 64, f32, torch.float8_e4m3fn, False, device="cpu").format == B.E4M3
    with pytest.raises(ValueError):
        B.KvBlocks(d, 32, bf)                                                  # nothing
    with pytest.raises(ValueError):
        B.KvBlocks(d, 32, bf, k=c.k)                                           # half of it
    with pytest.raises(ValueError):
        B.KvBlocks(d, 24, bf, bounds=c.bounds)
    with pytest.raises(TypeError):
        B.KvBlocks(d, 32, torch.float16, bounds=c.bounds)
    with pytest.raises(TypeError):
        B.KvBlocks(d, 32, f32, bounds=c.bounds)
    with pytest.raises(ValueError):
        B.KvBlocks(d, 64, bf, bounds=c.bounds)                                 # bounds of other blocks
    with pytest.raises(ValueError):
        B.KvBlocks(dims(B, batch=2, stride=120), 16, bf, bounds=c.bounds)      # stride
    with pytest.raises(ValueError):
        B.KvBlocks(d, 32, bf, bounds=c.bounds, page_table=torch.zeros(2, 8, dtype=torch.int32), page_size=16)
    with pytest.raises(TypeError):
        B.KvBlocks(d, 32, bf, bounds=c.bounds, page_table=torch.zeros(2, 4, dtype=torch.int64), page_size=32)
    with pytest.raises(TypeError):
        B.KvBlocks(d, 32, bf, c.k.to(torch.uint8), c.v, c.k_scale, c.v_scale, c.k_tail, c.v_tail)
    with pytest.raises(ValueError):
        B.KvBlocks(d, 32, bf, bounds=c.bounds.transpose(0, 1).contiguous().transpose(0, 1))
    x = torch.zeros(2, 2, 1, 128, dtype=bf)
    with pytest.raises(ValueError):
        B.kv8_append(d, c, x, x, 1)                                            # a cache in host memory
    with pytest.raises(ValueError):
        B.kv8_append(dims(B, batch=3), c, x, x, 1)                             # other dims
    for bad, err in ((x[:1], ValueError), (x.float(), TypeError)):
        with pytest.raises(err):
            B._arg(c, bad, "k_new", bf, x.numel())
    with pytest.raises(ValueError):
        B._arg(c, torch.zeros(2, 2, 128, 2, dtype=bf).transpose(2, 3), "k_new", bf, 2 * 2 * 2 * 128)


def test_the_plain_forms_themselves():
    """The float64 forms that the GPU tests compare with, against torch's own e4m3 and by hand."""
    val = R.e4m3_values()
    assert torch.equal(val, torch.arange(0x7f, dtype=torch.uint8).view(torch.float8_e4m3fn).double())
    x = torch.randn(4000, generator=torch.Generator().manual_seed(1)) * 100
    mid = ((val[1:] + val[:-1]) / 2).float()
    x = torch.cat([x, mid, -mid]).clamp(-448, 448)
    assert torch.equal(R.round_e4m3(x.double())[0], x.to(torch.float8_e4m3fn).double())
    q, s = R.quantise(torch.tensor([[127.0, 0.5, 1.5, -2.5]], dtype=torch.float64), "i8")
    assert q.tolist() == [[127, 0, 2, -2]] and float(s) == 1.0
    assert R.candidates(10, 20, 3) == (0, 0) and R.candidates(100, 20, 3) == (3, 80)
    assert R.tokens_of([0, 1], 40, 16, 20, 3) == list(range(3, 20))
