"""Decode steps over a cache in 8 bits as bench.py times them: the caches hold what was appended, and a step attends it."""
import pytest
import torch

import bench
from paper_2502_12665_amd import binding as B
from paper_2502_12665_amd import synth
from tests import kv_blocks_ref as R
from tests.test_gpu_kv_blocks import Case, gen

pytestmark = pytest.mark.gpu
D = 128


@pytest.mark.parametrize("fmt, shared", [("i8", False), ("e4m3", True)])
@pytest.mark.parametrize("ctx", [1024, 1003])
def test_steps_of_the_benchmark(fmt, shared, ctx):
    """Through the last block twice and a half: the sequence's first blocks stay, the last one is what has been appended, and each step's
    selection and output are those of the sequence up to its token."""
    wl = synth.WORKLOADS["c1_tiny"].replace(batch=2, ctx_len=ctx, top_k=96, window=40)
    codes = torch.int8 if fmt == "i8" else torch.float8_e4m3fn
    run = bench.BlockCacheSteps(torch, B, synth, wl, codes, shared)
    x = synth.make_decode_inputs(wl, device="cuda")
    k, v, q = (x[c].cpu() for c in ("k", "v", "q"))
    st, c = run.state, run.cache
    cos_w, sin_w = st.cos_win.cpu().double(), st.sin_win.cpu().double()
    assert run.first + run.tokens == ctx and run.first % 16 == 0
    lengths = []
    for i in range(run.tokens * 5 // 2):
        out = run.step(i)
        n = run.first + i % run.tokens + 1
        lengths.append(n)
        if i % run.tokens not in (0, 1, 9, run.tokens - 1):
            continue
        torch.cuda.synchronize()
        for b in range(2):
            s = R.Sequence(k[b, 0, :n], v[b, 0, :n], 16, fmt)
            full = n // 16
            for name in "kv":
                got = getattr(c, name)[b, 0].float().cpu().double().reshape(-1, 16, D)[:full]
                assert torch.equal(got, s.codes[name])
                assert torch.equal(getattr(c, name + "_scale")[b, 0].cpu().double()[:full], s.scales[name])
                assert torch.equal(getattr(c, name + "_tail")[b, 0].cpu()[: n % 16], (k if name == "k" else v)[b, 0, full * 16:n])
            assert torch.equal(c.bounds[b, 0].cpu().double()[: -(-n // 16)], s.bounds)
            q_rot = st.q_rot[b].cpu().double()
            picked = R.select(q_rot, s.bounds, n, 16, 40, wl.n_sink, 6, shared)
            for h in range(4):
                blocks = picked[0 if shared else h][0]
                assert st.block_idx[b, 0 if shared else h].tolist() == blocks
                want, off = R.attend(q[b, h].double(), q_rot[h], s.rows["k"], s.rows["v"], n, R.tokens_of(blocks, n, 16, 40, wl.n_sink), 40, wl.n_sink,
                                     cos_w, sin_w)
                err = (out[b, h].cpu().double() - want).abs()
                assert (err <= off + 2.0 ** -24 * want.abs()).all(), (i, b, h)
    assert lengths.count(ctx) == 2 and lengths.count(run.first + 1) == 3


@pytest.mark.parametrize("page", [0, 64])
@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
def test_a_sequence_may_go_back_to_the_beginning_of_a_block(fmt, page):
    """Other tokens from a block's border on: the cache is that of the sequence as it is now, bounds too."""
    c = Case([100, 77, 64], 4, 2, 32, fmt, "bf16", page, seed=7)
    c.append([90, 77, 64])
    for b, at in ((0, 64), (1, 32), (2, 0)):
        for x in (c.k, c.v):
            x[b][:, at:] = 0.25 * torch.randn(2, x[b].shape[1] - at, D, generator=gen(b)).to(c.dtype)
        c.have[b] = at
    c.append([65, 40, 64])
    for b, n in ((0, 65), (1, 40), (2, 64)):
        for kv in range(2):
            want, full = c.seq(b, kv, n), n // 32
            assert torch.equal(c.piece(c.cache.bounds, b, kv).double()[: -(-n // 32)], want.bounds)
            for x in "kv":
                assert torch.equal(c.piece(getattr(c.cache, x), b, kv).float().double().reshape(-1, 32, D)[:full], want.codes[x])
                assert torch.equal(c.piece(getattr(c.cache, x + "_scale"), b, kv).double()[:full], want.scales[x])
                assert torch.equal(getattr(c.cache, x + "_tail")[b, kv].cpu()[: n - full * 32], getattr(c, x)[b][kv, full * 32:n])
