"""Calls on a cache cut into blocks by every kernel that they have: heads, types, block sizes and numbers of blocks of which each takes a
path of its own."""
import pytest
import torch

from paper_2502_12665_amd import binding as B
from paper_2502_12665_amd import synth
from tests import kv_blocks_ref as R
from tests.test_gpu_kv_blocks import Case, check_attend, check_select, dims_of, draw_sel, gen, run_attend, run_select

pytestmark = pytest.mark.gpu
D = 128
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 6, 7, 8])
def test_attention_of_every_group_type_and_format(fmt, dtype, G):
    """A selection shared by G heads, tokens and blocks, with a window that ends inside a block."""
    c = Case([301, 64, 45], 2 * G, 2, 32, fmt, dtype, seed=100 + G, bounds=False)
    c.append(c.lens)
    for unit, n_sel in ((1, 150), (32, 5)):
        sel = draw_sel(c, unit, True, n_sel, 37, 2, 101)
        got = run_attend(c, sel, unit, True, 37, 2)
        check_attend(c, *got, sel, unit, True, 37, 2)


@pytest.mark.parametrize("fmt, dtype", [("i8", "f32"), ("i8", "bf16"), ("e4m3", "f32"), ("e4m3", "bf16")])
@pytest.mark.parametrize("G", [5, 6, 7, 8])
@pytest.mark.parametrize("window", [0, 1, 9])
def test_selected_rows_of_the_incomplete_block(fmt, dtype, G, window):
    """A selection shared by 5 to 8 heads, whose last tokens are still in the tail; sequences that have nothing else, too."""
    c = Case([64 + 61, 64, 50, 1, 128 + 17], G, 1, 64, fmt, dtype, seed=110 + G, bounds=False)
    c.append(c.lens)
    for unit, n_sel in ((1, 125), (64, 3)):
        sel = draw_sel(c, unit, True, n_sel, window, 3, 111)
        got = run_attend(c, sel, unit, True, window, 3)
        check_attend(c, *got, sel, unit, True, window, 3)


@pytest.mark.parametrize("heads, kv_heads, n_sel", [(5, 1, 1500), (8, 1, 3000), (14, 2, 2000)])
def test_shared_rows_of_the_incomplete_block_in_parts(heads, kv_heads, n_sel):
    """The same shared out among several workgroups: each has its own share of the selection and of the incomplete block's rows."""
    c = Case([3301, 90], heads, kv_heads, 128, "i8", "f32", seed=115, bounds=False)
    c.append(c.lens)
    sel = draw_sel(c, 1, True, n_sel, 11, 5, 116)
    for row in sel[0]:
        row[:100] = sorted(set(range(3290 - 90, 3290)) | set(row[:10]))[:100]   # (many of them in the tail, in one part's share)
        row[:] = list(dict.fromkeys(row))
    got = run_attend(c, sel, 1, True, 11, 5)
    check_attend(c, *got, sel, 1, True, 11, 5)


@pytest.mark.parametrize("fmt, dtype", [("i8", "f32"), ("i8", "bf16"), ("e4m3", "f32"), ("e4m3", "bf16")])
@pytest.mark.parametrize("G", [2, 4, 5, 8])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_one_head_of_a_shared_selection_that_is_not_finite(fmt, dtype, G, bad):
    """Its output is NaN; those of the heads that share its tile are what they are without it, bit for bit: far rows, window, tail."""
    c = Case([190, 96], 2 * G, 2, 32, fmt, dtype, seed=140 + G, bounds=False)
    c.append(c.lens)
    sel = draw_sel(c, 32, True, 3, 40, 1, 141)
    fine, q_rot = run_attend(c, sel, 32, True, 40, 1)[:2]
    wrong, q = q_rot.clone(), c.q.clone()
    wrong[0, 1, 77] = bad                                  # (far rows of one head, the window of another)
    c.q[1, G, 3] = bad
    got = run_attend(c, sel, 32, True, 40, 1, q_rot=wrong)[0]
    assert got[0, 1].isnan().all() and got[1, G].isnan().all()
    keep = torch.ones(2, 2 * G, dtype=torch.bool)
    keep[0, 1] = keep[1, G] = False
    assert torch.equal(got[keep], fine[keep])
    c.q = q
    # nothing but placeholders for a head that is not finite: zeros
    none = [[[], []], [[], []]]
    assert (run_attend(c, none, 32, True, 0, 0, q_rot=wrong)[0] == 0).all()


@pytest.mark.parametrize("blocks", [255, 256, 257, 1024, 1025, 2047, 2048, 2049, 3000, 4096])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_selection_on_either_side_of_its_kernels_borders(blocks, dtype):
    """Each number of blocks a thread has; the blocks of the last round are the best, so that what it leaves out would show."""
    blk, Hq, Hkv, ctx = 16, 4, 2, blocks * 16 - 3
    c = Case.__new__(Case)
    c.batch, c.heads, c.kv_heads, c.G, c.blk, c.page, c.dims = 2, Hq, Hkv, 2, blk, 0, dims_of(2, Hq, Hkv, ctx, blocks * 16)
    c.have = [ctx, ctx - 300]
    c.inv = synth.inv_freq(D, 500000.0)
    g = gen(blocks)
    c.q = torch.randn(2, Hq, D, generator=g).to(DT[dtype])
    mid = torch.randn(2, Hkv, blocks, D, generator=g) * 0.5
    wide = 2 + 2 * (torch.arange(blocks) >= blocks - 40).float()[:, None]
    bd = torch.stack([mid - wide, mid + wide], 3).to(DT[dtype])
    c.cache = B.KvBlocks(c.dims, blk, DT[dtype], bounds=bd.cuda())
    bounds = [[bd[b, kv, : -(-c.have[b] // blk)].double() for kv in range(Hkv)] for b in range(2)]
    for shared in (False, True):
        for top in (1, 60, 200):
            o = run_select(c, shared, top, 5, 20)
            check_select(c, o, shared, top, 5, 20, bounds=bounds)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("blk, page", [(16, 0), (16, 64), (32, 32), (64, 128), (128, 0), (128, 128), (128, 512)])
def test_bounds_alone(dtype, blk, page):
    """a2ats_key_bounds for every type and block size, contiguous and in pages, in pieces across block borders, sequences of their own."""
    c = Case([500, 129, 0, 1], 2, 2, blk, "i8", dtype, page, seed=120 + blk)
    cache = B.KvBlocks.empty(c.dims, blk, DT[dtype], codes=None, page_table=c.cache.page_table, page_size=page,
                             n_pages=c.cache.k.shape[0] if page else 0)
    cache.bounds.fill_(-77.0)
    have = [0, 0, 0, 0]
    for upto in ([1, 0, 0, 0], [blk - 1, 3, 0, 1], [blk + 1, blk, 0, 1], [300, 128, 0, 1], [500, 129, 0, 1]):
        m = [u - h for u, h in zip(upto, have)]
        new = torch.full((4, 2, max(m), D), 1e4, dtype=DT[dtype])
        for b in range(4):
            new[b, :, : m[b]] = c.k[b][:, have[b]:upto[b]]
        B.key_bounds(c.dims, cache, new.cuda(), max(m), *(torch.tensor(t, dtype=torch.int32, device="cuda") for t in (upto, m)))
        have = upto
        torch.cuda.synchronize()
        for b in range(4):
            for kv in range(2):
                got, used = c.piece(cache.bounds, b, kv).double(), -(-have[b] // blk)
                assert torch.equal(got[:used], c.seq(b, kv, have[b]).bounds), (b, kv, have)
                assert (got[used:] == -77).all()


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("heads, kv_heads, shared", [(4, 2, False), (7, 1, False), (7, 1, True), (8, 2, True)])
def test_tokens_that_the_codes_select(fmt, heads, kv_heads, shared):
    """a2ats_score_topk (or its shared form) over the code matrix, and its tokens attended from the cache in 8 bits: sequences of their own lengths."""
    n, K, w, sink, blk = 2000, 130, 50, 3, 32
    wl = synth.WORKLOADS["c1_tiny"].replace(batch=2, n_q_heads=heads, n_kv_heads=kv_heads, ctx_len=n, kv_dtype="bf16")
    x = synth.make_decode_inputs(wl, device="cuda")
    dims = B.make_dims(2, heads, kv_heads, D, wl.n_sub, n, -(-n // blk) * blk)
    codes = torch.zeros(2, kv_heads, dims.ctx_stride, wl.n_sub, dtype=x["codes"].dtype, device="cuda")
    codes[:, :, :n] = x["codes"]
    lens = torch.tensor([n, 1203], dtype=torch.int32, device="cuda")
    cache = B.KvBlocks.empty(dims, blk, torch.bfloat16, torch.int8 if fmt == "i8" else torch.float8_e4m3fn)
    B.kv8_append(dims, cache, x["k"], x["v"], n, lens)
    st = B.DecodeState(dims, K, w, sink, torch.bfloat16, x["inv_freq"], wl.wrope_b)
    lut = (B.build_lut_shared if shared else B.build_lut)
    lut(dims, x["q"], st.cos_b, st.sin_b, x["codebook"], st.q_rot, st.lut, st.lut_scale)
    H = kv_heads if shared else heads
    of = B.make_dims(2, H, kv_heads, D, wl.n_sub, n, dims.ctx_stride)        # (the shared selection is that of one head a KV head)
    idx = torch.empty(2, H, K, dtype=torch.int32, device="cuda")
    cnt = torch.empty(2, H, dtype=torch.int32, device="cuda")
    ws = torch.empty(max(B.workspace_bytes(of, B.OP_SCORE_TOPK, K, w), B.workspace_bytes(dims, B.OP_ATTN_KV8, K, w), 256), dtype=torch.uint8,
                     device="cuda")
    B.score_topk(of, codes, st.lut, st.lut_scale, K, w, sink, lens, idx, cnt, None, None, ws)
    out = torch.empty(2, heads, D, dtype=torch.bfloat16, device="cuda")
    B.sparse_attn_kv8(dims, cache, x["q"], st.q_rot, idx, cnt, K, 1, shared, w, sink, st.cos_win, st.sin_win, lens, out, ws)
    torch.cuda.synchronize()
    cos_w, sin_w = st.cos_win.cpu().double(), st.sin_win.cpu().double()
    for b, m in enumerate((n, 1203)):
        for h in range(heads):
            kv = h * kv_heads // heads
            s = R.Sequence(x["k"][b, kv, :m].cpu(), x["v"][b, kv, :m].cpu(), blk, fmt)
            at = kv if shared else h
            assert int(cnt[b, at]) == K
            pos = idx[b, at].tolist()
            assert len(set(pos)) == K and min(pos) >= sink and max(pos) < m - w
            want, off = R.attend(x["q"][b, h].cpu().double(), st.q_rot[b, h].cpu().double(), s.rows["k"], s.rows["v"], m, pos, w, sink, cos_w, sin_w)
            err = (out[b, h].cpu().double() - want).abs()
            assert (err <= off + 2.0 ** -8 * (want.abs() + off)).all(), (b, h, float(err.max()))


@pytest.mark.parametrize("shared, page, dtype, fmt, G", [(False, 0, "f32", "e4m3", 1), (True, 64, "bf16", "i8", 7), (True, 0, "f32", "i8", 5)])
def test_decode_steps_over_two_borders(shared, page, dtype, fmt, G):
    """61 tokens, one by one: the sequences complete two blocks each and end inside of one, every eleventh step and those about the borders
    compared with float64."""
    c = Case([190 + 61, 61], G, 1, 32, fmt, dtype, page, seed=130)
    c.append([190, 0])
    st = B.BlockDecodeState(c.dims, c.cache, 3, 20, 2, c.inv, 2048, shared)
    lens = torch.tensor([190, 0], dtype=torch.int32, device="cuda")
    steps = completed = checked = 0
    for i in range(61):
        lens += 1
        k, v = (torch.stack([t[b][:, (190, 0)[b] + i] for b in range(2)]).unsqueeze(2).contiguous().cuda() for t in (c.k, c.v))
        q = torch.randn(2, G, D, generator=gen(1000 + i)).to(c.dtype)
        out = st.step(q.cuda(), k, v, lens)
        c.have = [190 + i + 1, i + 1]
        steps += 1
        completed += sum(n % 32 == 0 for n in c.have)
        if i % 11 == 0 or any(n % 32 in (0, 1) for n in c.have):
            checked += 1
            c.q = q
            torch.cuda.synchronize()
            c.check_cache()
            o = {"q_rot": st.q_rot.cpu(), "idx": st.block_idx.cpu(), "count": st.block_count.cpu(), "score": st.block_score.cpu()}
            check_select(c, o, shared, 3, 20, 2)
            sel = [[[j for j in o["idx"][b, h].tolist() if j >= 0] for h in range(1 if shared else G)] for b in range(2)]
            check_attend(c, out.cpu(), o["q_rot"], st.cos_win.cpu().double(), st.sin_win.cpu().double(), sel, 32, shared, 20, 2)
    assert lens.tolist() == [251, 61] and (steps, completed) == (61, 3) and checked == 11
