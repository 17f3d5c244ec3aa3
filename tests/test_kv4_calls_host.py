"""Calls of the operators on a cache in 4 bits, and of the norms, that their documentation allows: host side.  No GPU."""
import pytest
import torch


@pytest.fixture(scope="module")
def B():
    from paper_2502_12665_amd import binding as b
    b.lib()
    return b


@pytest.mark.parametrize("batch", [1, 2, 4])
def test_layouts_of_no_tokens(B, batch):
    """Projections of no tokens, of a batch as of one sequence: nothing is refused (their strides say nothing)."""
    d = B.make_dims(batch, 8, 2, 128, 16, 100, 128)
    qkv = torch.zeros(batch, 5, 1536)
    for x in (torch.zeros(batch, 0, 1024), qkv[:, :0, :1024], torch.zeros(batch, 0, 8, 128), qkv[:, 2:2, :1024].unflatten(-1, (8, 128))):
        B._projected(d, x, "q", 8, 0)
    with pytest.raises(ValueError):
        B._projected(d, torch.zeros(batch, 0, 512), "q", 8, 0)


def takes(B, d, n_sel, size, window, shared, ws_bytes):
    """Whether the attention's call takes a workspace of so many bytes (queries that are missing are refused after it)."""
    c = B.Kv4Struct(16, 16, None, None, 0, 16, 1)
    rc = B.lib().a2ats_sparse_attn_kv4(d, c, None, None, None, None, n_sel, size, int(shared), window, 3, None, None, None, None,
                                       16 if ws_bytes else None, ws_bytes, None)
    assert rc in (-1, -3), rc
    return rc == -1


HEADS = [(1, 1), (8, 2), (28, 4), (32, 8), (64, 8)]


def test_workspaces_hold_every_plan(B):
    """What a2ats_workspace_bytes names for the most selected tokens and the widest window is enough for every call with fewer, of tokens as of
    blocks, shared or not."""
    some = 0
    for heads, kv_heads in HEADS:
        for batch in (1, 2, 5, 9, 16, 33, 36, 48, 49, 80, 112):
            for n in (90, 1000, 20000):
                d = B.make_dims(batch, heads, kv_heads, 128, 16, n, -(-n // 16) * 16)
                for most, wide in ((300, 0), (2048, 64), (4096, 700), (65536, 128)):
                    need = B.workspace_bytes(d, B.OP_ATTN_KV4, most, wide)
                    some += need > 0
                    for rows in (0, 1, 65, 257, 300, 600, 2048, 4096, 16384, 65536):
                        for w in (0, 1, 64, 128, 700):
                            if rows > most or w > wide:
                                continue
                            for shared in (False, True):
                                n_sel, size = (rows, 1) if rows <= 4096 else (rows // 16, 16)
                                assert takes(B, d, n_sel, size, w, shared, need), (heads, batch, n, most, wide, rows, w, shared)
    assert some > 100


def least(B, problems, rows, window, shared):
    """The workspace that a call of so many heads (or of KV heads with four heads each) asks for, in parts of a head's state; 1: none."""
    d = B.make_dims(problems, 4 if shared else 1, 1, 128, 16, 1 << 17, 1 << 17)
    n_sel, size = (rows, 1) if rows <= 4096 else (rows // 16, 16)
    state = d.batch * d.n_q_heads * 130 * 4
    if takes(B, d, n_sel, size, window, shared, 0):
        return 1
    return next(p for p in range(2, 13) if takes(B, d, n_sel, size, window, shared, p * state))


@pytest.mark.parametrize("shared, rows", [(False, 4096), (False, 16000), (True, 8000), (True, 16000)])
def test_parts_go_by_ranges_of_sizes(B, shared, rows):
    """Problems around those that leave half a round of CUs over: the same plan as their neighbours, not one for exact numbers."""
    for lo, hi, parts in ((129, 256, 1), (257, 384, 2), (385, 512, 1), (513, 640, 2), (641, 768, 1), (769, 896, 2), (897, 1024, 1)):
        for problems in (lo, lo + 1, (lo + hi) // 2, hi - 1, hi):
            assert least(B, problems, rows, 64, shared) == parts, (problems, parts)
            assert least(B, problems, 300, 64, shared) == 1
    for problems, parts in ((1, 12), (2, 12), (21, 12), (32, 8), (64, 4), (128, 2)):
        assert least(B, problems, 65536, 64, shared) <= parts
