"""Which appends are refused for their size: launches of 2^32 threads, of as many as are launched.  Nothing is launched here: a call
that is not too large is refused for its new keys without an address."""
import ctypes

import pytest

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
