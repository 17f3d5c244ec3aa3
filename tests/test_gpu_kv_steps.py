"""Decode steps over a cache in 8 bits as bench.py times them: the caches hold what was appended, and a step attends it."""
import os
import re

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


def test_the_readme_program():
    """README.md's code blocks as they stand, behind each other: the tokens that the codes select attended from the 8-bit cache, then 20 generated
    tokens, after which the cache holds the prompt and all of them."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = "\n".join(re.findall(r"```python\n(.*?)```", open(os.path.join(root, "README.md")).read(), re.S))
    at = code.index("# or blocks selected")
    env = {}
    exec(code[:at], env)
    wl, x, st, cache, grown = (env[n] for n in ("wl", "x", "st", "cache", "grown"))
    N, w, G = wl.ctx_len, wl.window, wl.n_q_heads // wl.n_kv_heads
    torch.cuda.synchronize()
    bs, first = env["bs"], env["out"].cpu()
    cos_w, sin_w = bs.cos_win.cpu().double(), bs.sin_win.cpu().double()

    def attended(out, h, k, v, q, q_rot, n, positions):
        s = R.Sequence(k, v, 16, "i8")
        want, off = R.attend(q.double(), q_rot.double(), s.rows["k"], s.rows["v"], n, positions, w, 0, cos_w, sin_w)
        err = (out.double() - want).abs()
        assert (err <= off + 2.0 ** -8 * (want.abs() + off)).all(), (h, float(err.max()))
        return s

    for h in (0, wl.n_q_heads - 1):
        assert int(st.topk_count[0, h]) == wl.top_k
        attended(first[0, h], h, x["k"][0, h // G].cpu(), x["v"][0, h // G].cpu(), x["q"][0, h].cpu(), st.q_rot[0, h].cpu(), N,
                 st.topk_idx[0, h].tolist())
    g = gen(1)
    new = [[torch.randn(1, n, D, generator=g).bfloat16() for n in (wl.n_q_heads, wl.n_kv_heads, wl.n_kv_heads)] for _ in range(20)]
    env["tokens"] = [(q.cuda(), k.unsqueeze(2).cuda(), v.unsqueeze(2).cuda()) for q, k, v in new]
    exec(code[at:], env)
    torch.cuda.synchronize()
    n = N + 20
    assert env["seq_lens"].tolist() == [n] and grown.ctx_len >= n
    for h in (0, wl.n_q_heads - 1):
        kv = h // G
        k, v = (torch.cat([x[c][0, kv].cpu()] + [t[i][0, kv:kv + 1] for t in new]) for c, i in (("k", 1), ("v", 2)))
        blocks = [c for c in bs.block_idx[0, h].tolist() if c >= 0]
        assert len(blocks) == wl.top_k // 16
        s = attended(env["out"][0, h].cpu(), h, k, v, new[-1][0][0, h], bs.q_rot[0, h].cpu(), n, R.tokens_of(blocks, n, 16, w, 0))
        assert R.select(bs.q_rot[0, h:h + 1].cpu().double(), s.bounds, n, 16, w, 0, len(blocks), False)[0][0] == blocks
        assert torch.equal(cache.k[0, kv].float().cpu().double().reshape(-1, 16, D)[: n // 16], s.codes["k"])
        assert torch.equal(cache.v_tail[0, kv, : n % 16].cpu(), v[n // 16 * 16:])
