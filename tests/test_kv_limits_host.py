"""Sizes of calls on a cache cut into blocks: appends that are refused for launches of 2^32 threads, of as many as are launched, and the
workspaces that selections and attention ask for.  Nothing is launched here: a call whose size passes is refused for new keys or
queries without an address."""
import ctypes

import pytest
import torch

ONE = 16


@pytest.fixture(scope="module")
def B():
    from paper_2502_12665_amd import binding as b
    b.lib()
    return b


def struct(B, block):
    f = dict(k=ONE, v=ONE, k_scale=ONE, v_scale=ONE, k_tail=ONE, v_tail=ONE, bounds=ONE, page_table=None, page_size=0, block=block, format=0,
             kv_dtype=1)
    return B.KvBlocksStruct(*[f[x[0]] for x in B.KvBlocksStruct._fields_])


N = 1 << 20


@pytest.mark.parametrize("block, slab, threads", [(16, 64, 256), (32, 64, 256), (64, 64, 256), (128, 128, 512)])
@pytest.mark.parametrize("rows", [True, False])
def test_appends(B, block, slab, threads, rows):
    """A workgroup for each slab of 64 or 128 rows from the beginning of a block on, of keys and (if there are rows) of values."""
    parts = (N + block - 1 + slab - 1) // slab * (2 if rows else 1)
    largest = ((1 << 32) - 1) // (parts * threads)
    for batch, rc in ((largest, -1), (largest + 1, -2)):
        d, c = B.make_dims(batch, 1, 1, 128, 16, N, N), struct(B, block)
        if rows:
            assert B.lib().a2ats_kv8_append(ctypes.byref(d), ctypes.byref(c), None, ONE, N, None, None, None) == rc, batch
        else:
            assert B.lib().a2ats_key_bounds(ctypes.byref(d), ctypes.byref(c), None, N, None, None, None) == rc, batch


def least(call):
    """The least workspace with which `call` gets past its check."""
    lo, hi = 0, 1 << 40
    assert call(hi) == -1
    if call(0) == -1:
        return 0
    while hi - lo > 1:
        mid = (lo + hi) // 2
        rc = call(mid)
        assert rc in (-1, -3)
        lo, hi = (mid, hi) if rc == -3 else (lo, mid)
    return hi


SHAPES = [(1, 4, 1, 64), (1, 32, 8, 32768), (2, 28, 4, 131072), (4, 32, 8, 5000), (16, 32, 8, 32768), (32, 64, 8, 999), (1, 8, 8, N)]


@pytest.mark.parametrize("batch, heads, kv_heads, n", SHAPES)
def test_the_workspace_figure_of_selections(B, batch, heads, kv_heads, n):
    """One figure for every block size and both kinds of selection."""
    d = B.make_dims(batch, heads, kv_heads, 128, 16, n, -(-n // 128) * 128)
    figure, most = B.workspace_bytes(d, B.OP_BLOCK_TOPK), 0
    for block in (16, 32, 64, 128):
        for shared in (0, 1):
            for top in (0, 1, 4096):
                c = struct(B, block)
                need = least(lambda n_ws: B.lib().a2ats_block_topk(ctypes.byref(d), ctypes.byref(c), None, ONE, ONE, ONE, shared, top, 8, 3, None, ONE,
                                                                   ONE, None, None, None, ONE, n_ws, None))
                blocks, H = -(-n // block), kv_heads if shared else heads
                assert batch * H * blocks * 4 <= need <= figure                # (a score for each head and block)
                most = max(most, need)
    assert most == figure


@pytest.mark.parametrize("batch, heads, kv_heads, n", SHAPES)
@pytest.mark.parametrize("window", [0, 64, 700])
def test_the_workspace_figure_of_attention(B, batch, heads, kv_heads, n, window):
    """n_sel * sel_size says it for both units, both kinds of selection, and any number of sinks."""
    d = B.make_dims(batch, heads, kv_heads, 128, 16, n, -(-n // 128) * 128)
    parts = set()
    for block, size, n_sel in ((16, 1, 0), (16, 1, 1), (16, 1, 300), (64, 1, 2048), (32, 1, 4096), (16, 16, 20), (32, 32, 64), (128, 128, 9),
                               (64, 64, 500), (128, 128, 4096)):
        figure, most = B.workspace_bytes(d, B.OP_ATTN_KV8, n_sel * size, window), 0
        for shared in (0, 1):
            for sink in (0, 4, 64, 5000):
                c = struct(B, block)
                need = least(lambda n_ws: B.lib().a2ats_sparse_attn_kv8(ctypes.byref(d), ctypes.byref(c), None, ONE, ONE, ONE, n_sel, size, shared,
                                                                        window, sink, ONE, ONE, None, ONE, ONE, n_ws, None))
                assert need <= figure and need % (batch * heads * 130 * 4) == 0   # (parts of 128 sums, a maximum and a sum)
                parts.add(need // (batch * heads * 130 * 4))
                most = max(most, need)
        assert most == figure
    assert parts <= {0} | set(range(2, 13))


def test_caches_of_blocks_that_there_are_not(B):
    """Refused before anything is allocated."""
    d = B.make_dims(2, 4, 2, 128, 16, 100, 128)
    table = torch.zeros(2, 4, dtype=torch.int32)
    for kw, err in ((dict(block=0), ValueError), (dict(block=24), ValueError), (dict(block=256), ValueError), (dict(kv_dtype=torch.float16), TypeError),
                    (dict(page_table=table, page_size=0, n_pages=8), ValueError), (dict(page_table=table, page_size=48, n_pages=8), ValueError)):
        with pytest.raises(err):
            B.KvBlocks.empty(d, **{"block": 32, "kv_dtype": torch.bfloat16, "device": "nowhere", **kw})
    with pytest.raises(ValueError):
        B.KvBlocks.empty(B.make_dims(2, 4, 2, 128, 16, 100, 100), 16, torch.bfloat16, device="nowhere")
