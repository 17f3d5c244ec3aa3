"""Calls of the operators on a cache in 4 bits, and of the norms, that their documentation allows and that lie beside the ordinary ones,
against plain float64 forms, through the C ABI."""
import pytest
import torch

from paper_2502_12665_amd import binding as B
from tests.test_gpu_kv4 import Case, check_attend, draw_sel, gen, run_attend

pytestmark = pytest.mark.gpu
D = 128


@pytest.mark.parametrize("batch", [1, 4])
def test_norms_of_no_tokens(batch):
    """n_new 0 is a no-op, of a batch too."""
    dims = B.make_dims(batch, 8, 2, D, 16, 100, 128)
    qkv = torch.zeros(batch, 0, 12 * D, device="cuda")
    out = torch.empty(batch, 8, 0, D, device="cuda")
    B.qk_norm_rope(dims, qkv[..., : 8 * D], qkv[..., 8 * D: 10 * D], 0, None, None, 1e-6, None, None, q_norm=out,
                   k_norm=torch.empty(batch, 2, 0, D, device="cuda"))
    torch.cuda.synchronize()


@pytest.mark.parametrize("G, shared", [(1, False), (4, False), (3, True), (7, True)])
@pytest.mark.parametrize("q_at, k_at", [(5, 70), (5, 69), (69, 5), (100, 3)])
def test_window_of_large_elements_that_do_not_meet(G, shared, q_at, k_at):
    """A query and keys of 2^100 each, in different elements, also in two of a pair that is not turned (the last token's never is): no
    product that counts is beyond float32, the logits are 0 and the output is the mean of the values, exactly (sums of few bits)."""
    c = Case([8], G, 1, 16, "f32", seed=101, bounds=False)
    c.inv = torch.zeros(64, dtype=torch.float64)            # (no rotation)
    c.k[0] = torch.zeros(1, 8, D)
    c.k[0][:, :, k_at] = 2.0 ** 100
    c.append(c.lens)
    c.q = torch.zeros(1, G, D)
    c.q[..., q_at] = 2.0 ** 100
    got = run_attend(c, [[[] for _ in range(1 if shared else G)]], 1, shared, 8, 0, q_rot=c.q)[0]
    want = c.seq(0, 0)[3].mean(0)
    assert torch.equal(got[0].double(), want.expand(G, D))


@pytest.mark.parametrize("four_bits", [True, False])
def test_steps_of_packed_projections(four_bits):
    """Queries, keys and values of a step as slices of one projection: the cache, the selection and the output are those of a step that is
    given them contiguous."""
    batch, heads, kv_heads = 3, 8, 2
    dims = B.make_dims(batch, heads, kv_heads, D, 16, 100, 112)
    inv = torch.exp(-torch.arange(64, dtype=torch.float64) / 8)
    g = gen(102)
    w = [(1 + 0.2 * torch.randn(D, generator=g)).cuda() for _ in range(2)]
    states = []
    for _ in range(2):
        cache = (B.Kv4Cache if four_bits else B.KvBlocks).empty(dims, 16, torch.bfloat16)
        cache.bounds.zero_()
        states.append((cache, B.BlockDecodeState(dims, cache, 2, 20, 1, inv, 64, False, q_weight=w[0], k_weight=w[1])))
    lens = torch.zeros(batch, dtype=torch.int32, device="cuda")
    for i in range(40):
        lens += 1
        x = torch.randn(batch, heads + 2 * kv_heads, D, generator=g).bfloat16().cuda()
        q, k, v = x[:, :heads], x[:, heads:heads + kv_heads].unsqueeze(2), x[:, heads + kv_heads:].unsqueeze(2)
        outs = [states[0][1].step(q, k, v, lens), states[1][1].step(q.contiguous(), k.contiguous(), v.contiguous(), lens)]
        assert torch.equal(*outs) and torch.equal(states[0][1].block_idx, states[1][1].block_idx), i
    # (codes of 8 bits: of the two complete blocks, the others are not written)
    for name, n in (("rows", 40), ("scales", 40)) if four_bits else (("k", 32), ("v", 32), ("k_scale", 2), ("v_scale", 2), ("v_tail", 16)):
        assert torch.equal(*(getattr(s[0], name)[:, :, :n].contiguous().view(torch.uint8) for s in states)), name
    assert torch.isfinite(outs[0]).all() and (outs[0] != 0).any()
    for bad in (v.float(), v[:, :1], v.transpose(0, 1)):    # (neither converted nor spread)
        with pytest.raises((TypeError, ValueError)):
            states[0][1].step(q, k, bad, lens)


def needs_parts(c, n_sel, size, shared, window):
    """Whether the call is one of several workgroups a head: it is refused without a workspace."""
    o = torch.zeros(c.batch, c.heads, D, dtype=c.dtype, device="cuda")
    H = c.kv_heads if shared else c.heads
    idx, cnt = (torch.zeros(c.batch, H, n, dtype=torch.int32, device="cuda") for n in (n_sel, 1))
    tables = [torch.zeros(max(window, 1), D // 2, device="cuda")] * 2
    if B.workspace_bytes(c.dims, B.OP_ATTN_KV4, n_sel * size, window) == 0:
        return False
    try:
        B.sparse_attn_kv4(c.dims, c.cache, o, o.float(), idx, cnt, n_sel, size, shared, window, 0, *tables, None, torch.zeros_like(o), None)
    except B.A2atsError as e:
        assert "orkspace" in str(e), e
        return True
    return False


@pytest.mark.parametrize("page", [0, 64])
@pytest.mark.parametrize("unit, n_sel, window, n_sink", [(1, 1500, 100, 4), (32, 50, 300, 0), (1, 1024, 0, 1200)])
@pytest.mark.parametrize("G, shared", [(1, False), (4, False), (8, False), (1, True), (3, True), (8, True)])
def test_parts_of_ragged_batches(G, shared, unit, n_sel, window, n_sink, page):
    """Several workgroups a head over sequences of 5000 tokens to none: parts without a row, selections split inside of a block, windows and
    sinks past the sequence's end."""
    c = Case([900, 5000, 70, 0, 1, 2100], 2 * G, 2, 32, "bf16" if G % 4 else "f32", page, seed=110 + G, bounds=False)
    c.append(c.lens)
    assert needs_parts(c, n_sel, unit, shared, window)
    sel = draw_sel(c, unit, shared, n_sel, window, n_sink, 111)
    got = run_attend(c, sel, unit, shared, window, n_sink)
    check_attend(c, *got, sel, unit, shared, window, n_sink)
    assert (got[0][3] == 0).all()


@pytest.mark.parametrize("G, kv_heads, shared, unit, n_sel", [(4, 2, False, 1, 4096), (1, 8, False, 16, 260), (2, 8, True, 16, 380)])
@pytest.mark.parametrize("page", [0, 32])
def test_two_parts_of_many_heads(G, kv_heads, shared, unit, n_sel, page):
    """More heads (KV heads) than compute units, half a round of them left over: two workgroups each."""
    lens = [6300] + [17, 0, 300, 1, 65] * 7
    c = Case(lens, kv_heads * G, kv_heads, 16, "bf16", page, seed=115, bounds=False)
    assert 256 < c.batch * (kv_heads if shared else c.heads) <= 384
    c.append(c.lens)
    assert needs_parts(c, n_sel, unit, shared, 64)
    sel = draw_sel(c, unit, shared, n_sel, 64, 2, 116)
    got = run_attend(c, sel, unit, shared, 64, 2)
    check_attend(c, *got, sel, unit, shared, 64, 2)
