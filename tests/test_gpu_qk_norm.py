"""Norms of queries and keys with their rotation (a2ats_qk_norm_rope) against the plain float64 form, and decode steps of a model that
has them over caches in 4 and 8 bits."""
import math

import pytest
import torch

from paper_2502_12665_amd import binding as B
from paper_2502_12665_amd import synth
from tests import kv4_ref as F
from tests import kv_blocks_ref as R
from tests.test_gpu_kv4 import Case, check_attend, gen

pytestmark = pytest.mark.gpu
D = 128
U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
ALL = ("q_norm", "k_norm", "q_pos", "k_pos")


def tables(n):
    inv = synth.inv_freq(D, 10000.0)
    _, _, cos, sin = B.rope_tables(D, inv, 0, n, "cuda")
    return cos, sin


def run(dims, q, k, n_new, qw, kw, eps, lens=None, news=None, want=ALL, table=None):
    dt = (q if q is not None else k).dtype
    heads = {"q": dims.n_q_heads, "k": dims.n_kv_heads}
    o = {x: torch.full((dims.batch, heads[x[0]], n_new, D), 7.0, dtype=dt, device="cuda") for x in want}
    cos, sin = table if table is not None else (tables(dims.ctx_len) if any("pos" in x for x in want) else (None, None))
    ints = [None if t is None else torch.tensor(t, dtype=torch.int32, device="cuda") for t in (lens, news)]
    B.qk_norm_rope(dims, q, k, n_new, None if qw is None else qw.cuda(), None if kw is None else kw.cuda(), eps, cos, sin, *ints, **o)
    torch.cuda.synchronize()
    return {x: t.cpu() for x, t in o.items()}, None if cos is None else (cos.cpu().double(), sin.cpu().double())


def check(dims, q, k, n_new, qw, kw, eps, lens, news, got, table):
    """q, k [B, n_new, H, D] on the host."""
    for x, o in got.items():
        src, w = ((q, qw), (k, kw))[x[0] == "k"]
        for b in range(dims.batch):
            n = dims.ctx_len if lens is None else min(max(lens[b], 0), dims.ctx_len)
            m = max(0, min(n_new if news is None else news[b], n_new, n))
            assert (o[b, :, m:] == 7).all(), (x, b)
            y = F.norm(src[b, :m].double(), w, eps).transpose(0, 1)                # [H, m, D]
            tol = F.NORM_ROUNDINGS * U * y.abs()
            if "pos" in x:
                cos, sin = table[0][n - m:n], table[1][n - m:n]
                a = y.abs()
                tol = F.ROTATED_ROUNDINGS * U * torch.cat([a[..., :64] * cos.abs() + a[..., 64:] * sin.abs(),
                                                           a[..., 64:] * cos.abs() + a[..., :64] * sin.abs()], -1)
                y = R.rotate(y, cos, sin)
            tol = tol + F.half_step(y.abs() + tol, o.dtype)
            err = (o[b, :, :m].double() - y).abs()
            assert (err <= tol).all(), (x, b, float((err / tol).max()))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads, kv_heads, packed", [(1, 1, True), (32, 8, True), (28, 4, False), (6, 3, True), (64, 8, False)])
@pytest.mark.parametrize("n_new", [1, 5, 70])
def test_norms(dtype, heads, kv_heads, packed, n_new):
    """Sequences of every length around n_new, with and without numbers of new tokens; slices of a projection and tensors of their own."""
    batch, ctx = 5, 90
    dims = B.make_dims(batch, heads, kv_heads, D, 16, ctx, ctx)
    g = gen(heads + n_new)
    qkv = (torch.randn(batch, n_new, (heads + 2 * kv_heads) * D, generator=g) * torch.exp2(torch.randint(-9, 9, (batch, n_new, 1), generator=g).float())).to(DT[dtype])
    q, k = qkv[..., : heads * D], qkv[..., heads * D:(heads + kv_heads) * D]
    on = qkv.cuda()
    dev = [on[..., : heads * D], on[..., heads * D:(heads + kv_heads) * D]]
    if not packed:
        dev = [t.contiguous() for t in dev]
    qw, kw = 1 + 0.3 * torch.randn(D, generator=g), torch.randn(D, generator=g)
    hq, hk = q.unflatten(-1, (heads, D)), k.unflatten(-1, (kv_heads, D))
    for lens, news in (([90, n_new, 1, 0, 33], None), ([90, 80, 100, -4, 3], [1, n_new, 200, 2, -1]), (None, None)):
        got, table = run(dims, *dev, n_new, qw, kw, 1e-6, lens, news)
        check(dims, hq, hk, n_new, qw, kw, 1e-6, lens, news, got, table)


@pytest.mark.parametrize("want", [("q_norm",), ("k_norm",), ("q_pos", "k_norm", "k_pos"), ("q_norm", "k_norm"), ("k_pos",), ("q_norm", "q_pos")])
def test_outputs_that_are_asked_for(want):
    """Queries or keys alone, without weights, one output or several: those that are made are the same as in a call for all."""
    dims = B.make_dims(2, 20, 4, D, 16, 40, 40)
    g = gen(3)
    q, k = torch.randn(2, 9, 20 * D, generator=g).bfloat16().cuda(), torch.randn(2, 9, 4 * D, generator=g).bfloat16().cuda()
    full, _ = run(dims, q, k, 9, None, None, 1e-5, [40, 20])
    has = {x[0] for x in want}
    got, _ = run(dims, q if "q" in has else None, k if "k" in has else None, 9, None, None, 1e-5, [40, 20], want=want)
    for x in want:
        assert torch.equal(got[x], full[x]), x
    check(dims, q.cpu().unflatten(-1, (20, D)), k.cpu().unflatten(-1, (4, D)), 9, None, None, 1e-5, [40, 20], None, full,
          [t.cpu().double() for t in tables(40)])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_any_size(dtype):
    """Rows of zeros, of the least and of the largest numbers, and of one element: no square overflows or is lost beside eps."""
    dt = DT[dtype]
    big = torch.finfo(dt).max
    x = torch.zeros(1, 12, D)
    g = gen(4)
    r = torch.randn(12, D, generator=g)
    for i, s in enumerate((0.0, 2.0 ** -126, 2.0 ** -80, 2.0 ** -40, 2.0 ** -10, 2.0 ** 20, 2.0 ** 70, 2.0 ** 120)):
        x[0, i] = r[i] * s
    x[0, 8, 5] = big
    x[0, 9] = big
    x[0, 10, 127] = -(2.0 ** -100)
    x[0, 11, ::2] = 2.0 ** 63
    x = x.to(dt)
    dims = B.make_dims(1, 1, 1, D, 16, 12, 12)
    for eps in (1e-6, 2.0 ** -126, 1.0):
        got, table = run(dims, x.cuda(), None, 12, None, None, eps, want=("q_norm", "q_pos"))
        check(dims, x[:, :, None], None, 12, None, None, eps, None, None, got, table)


def test_rows_that_are_not_finite():
    """They are not finite afterwards, and the rows beside them are what they would be."""
    dims = B.make_dims(1, 8, 2, D, 16, 3, 3)
    q, k = torch.randn(1, 3, 8 * D, generator=gen(5)), torch.randn(1, 3, 2 * D, generator=gen(6))
    clean, _ = run(dims, q.cuda(), k.cuda(), 3, None, None, 1e-6)
    q[0, 1, 2 * D + 7], k[0, 2, D + 100] = math.inf, math.nan
    got, _ = run(dims, q.cuda(), k.cuda(), 3, None, None, 1e-6)
    for x in got:
        h, t = (2, 1) if x[0] == "q" else (1, 2)
        assert not torch.isfinite(got[x][0, h, t]).all() and torch.isnan(got[x][0, h, t, 7 if x[0] == "q" else 100])
        got[x][0, h, t] = clean[x][0, h, t]
        assert torch.equal(got[x], clean[x])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_do_not_depend_on_their_neighbours(dtype):
    """Heads of a token beside others whose squares overflow, vanish or are not finite: the same bits as alone."""
    dims, g = B.make_dims(1, 16, 4, D, 16, 64, 64), gen(41)
    w = 1 + 0.2 * torch.randn(D, generator=g)
    x = torch.randn(1, 6, 20, D, generator=g).to(DT[dtype])
    y, at = x.clone(), torch.arange(20) % 4
    for head, scale in ((1, 2.0 ** 90), (2, 2.0 ** -90), (3, math.nan)):
        y[:, :, at == head] *= scale
    for eps in (1e-6, 2.0 ** -126):
        alone, beside = (run(dims, t[:, :, :16], t[:, :, 16:], 6, w, w, eps, [40], None)[0] for t in (x.cuda(), y.cuda()))
        for name, o in alone.items():
            assert torch.equal(o[:, 0::4], beside[name][:, 0::4]), name
            assert beside[name][:, 3::4].isnan().all()


def test_norms_over_32_bits_of_elements():
    """A projection of more than 2^31 elements, of which the last tokens are taken: offsets of 64 bits."""
    n, wide = 70000, 40 * D * 8                            # 2.9e9 bfloat16 elements
    dims = B.make_dims(1, 32, 8, D, 16, n, n)
    qkv = torch.zeros(1, n, wide, dtype=torch.bfloat16, device="cuda")
    x = torch.randn(3, 40 * D, generator=gen(7)).bfloat16()
    qkv[0, -3:, : 40 * D] = x.cuda()
    k_norm = torch.full((1, 8, n, D), 7.0, dtype=torch.bfloat16, device="cuda")
    B.qk_norm_rope(dims, None, qkv[..., 32 * D: 40 * D], n, None, None, 1e-6, None, None, k_norm=k_norm)
    got = {"k_norm": k_norm[:, :, -3:].cpu()}
    check(B.make_dims(1, 32, 8, D, 16, 3, 3), None, x[None, :, 32 * D:].unflatten(-1, (8, D)), 3, None, None, 1e-6, None, None, got, None)
    assert (k_norm[:, :, :-3] == 0).all()


# ---------------------------------------------------------------------------------------------- the operators together

@pytest.mark.parametrize("dtype, shared, page", [("bf16", False, 0), ("f32", True, 64), ("bf16", True, 32)])
def test_prompt_and_steps_together(dtype, shared, page):
    """A prompt is normalised and cached in 4 bits, its rotated keys are those of its positions; then steps: norm, append, selection of
    blocks, attention.  Each call is compared with the plain form of what the call before it wrote."""
    batch, heads, kv_heads, blk, ctx, top, window, n_sink = 2, 8, 2, 32, 200, 3, 20, 2
    c = Case([0] * batch, heads, kv_heads, blk, dtype, page, seed=11, ctx=ctx)
    dt = c.dtype
    g = gen(12)
    qw, kw = 1 + 0.2 * torch.randn(D, generator=g), 1 + 0.2 * torch.randn(D, generator=g)
    prompt = [150, 97]
    qkv = torch.randn(batch, 150, (heads + 2 * kv_heads) * D, generator=g).to(dt)
    q, k, v = (t.unflatten(-1, (-1, D)) for t in qkv.split([heads * D, kv_heads * D, kv_heads * D], -1))
    on = qkv.cuda()
    got, table = run(c.dims, on[..., : heads * D], on[..., heads * D:(heads + kv_heads) * D], 150, qw, kw, 1e-6, prompt, want=ALL)
    check(c.dims, q, k, 150, qw, kw, 1e-6, prompt, None, got, table)
    c.k = [got["k_norm"][b][:, : prompt[b]] for b in range(batch)]
    c.v = [v[b].transpose(0, 1)[:, : prompt[b]].contiguous() for b in range(batch)]
    lens = torch.tensor(prompt, dtype=torch.int32, device="cuda")
    B.kv4_append(c.dims, c.cache, got["k_norm"].cuda(), v.transpose(1, 2).contiguous().cuda(), 150, lens)
    c.have = list(prompt)
    c.check_cache()
    back = torch.empty(batch, kv_heads, 150, D, dtype=dt, device="cuda")
    B.kv4_read(c.dims, c.cache, 150, lens, None, back, None)
    for b in range(batch):
        for kv in range(kv_heads):
            assert torch.equal(back[b, kv, : prompt[b]].cpu().double(), c.seq(b, kv)[2])
    st = B.BlockDecodeState(c.dims, c.cache, top, window, n_sink, c.inv, 2048, shared, q_weight=qw.cuda(), k_weight=kw.cuda(), eps=1e-6)
    for i in range(40):
        x = torch.randn(batch, (heads + 2 * kv_heads), D, generator=g).to(dt)
        qn, kn, vn = x[:, :heads], x[:, heads:heads + kv_heads, None], x[:, heads + kv_heads:, None].contiguous()
        lens += 1
        out = st.step(qn.contiguous().cuda(), kn.contiguous().cuda(), vn.cuda(), lens).cpu()
        c.have = [h + 1 for h in c.have]
        o = {"q_norm": st.q_norm.cpu()[:, :, None], "k_norm": st.k_norm.cpu()}
        check(c.dims, qn[:, None], kn.transpose(1, 2), 1, qw, kw, 1e-6, c.have, None, o, None)
        c.q = st.q_norm.cpu()
        c.k = [torch.cat([a, b], 1) for a, b in zip(c.k, o["k_norm"])]
        c.v = [torch.cat([a, b], 1) for a, b in zip(c.v, vn)]
        c.rounded.clear()
        if i % 8 and i < 32:
            continue
        c.check_cache()
        q_rot, sel = st.q_rot.cpu(), []
        H = kv_heads if shared else heads
        for b in range(batch):
            sel.append([])
            for h in range(H):
                G = heads // kv_heads
                kv = h if shared else h // G
                qs = q_rot[b, h * G:(h + 1) * G] if shared else q_rot[b, h:h + 1]
                want = R.select(qs.double(), F.bounds(c.k[b][kv], blk), c.have[b], blk, window, n_sink, top, shared)[0][0]
                have = [j for j in st.block_idx[b, h].tolist() if j >= 0]
                assert have == want, (b, h)
                sel[b].append(have)
        check_attend(c, out, q_rot, st.cos_win.cpu().double(), st.sin_win.cpu().double(), sel, blk, shared, window, n_sink)


@pytest.mark.parametrize("four_bits", [True, False])
def test_captured_steps_replay(four_bits):
    """A step in a graph, replayed with other inputs and lengths, with eager work in between: every replay is the eager result."""
    dims = B.make_dims(2, 8, 2, D, 16, 300, 304)
    inv = synth.inv_freq(D, 500000.0)
    g = gen(20)
    w = [(1 + 0.2 * torch.randn(D, generator=g)).cuda() for _ in range(2)]

    def state():
        if four_bits:
            cache = B.Kv4Cache.empty(dims, 16, torch.bfloat16)
        else:
            cache = B.KvBlocks.empty(dims, 16, torch.bfloat16)
        cache.bounds.zero_()
        x = torch.randn(2, 2, 200, D, generator=gen(21)).bfloat16().cuda()
        lens = torch.tensor([200, 130], dtype=torch.int32, device="cuda")
        (B.kv4_append if four_bits else B.kv8_append)(dims, cache, x, x, 200, lens)
        return cache, B.BlockDecodeState(dims, cache, 4, 24, 1, inv, 2048, False, q_weight=w[0], k_weight=w[1])

    (cache, st), (other, se), (_, warm) = state(), state(), state()
    q = torch.zeros(2, 8, D, dtype=torch.bfloat16, device="cuda")
    k, v = (torch.zeros(2, 2, 1, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lens = torch.tensor([200, 130], dtype=torch.int32, device="cuda")
    warm.step(q, k, v, lens)                                # (the kernels are loaded before the capture)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        st.step(q, k, v, lens)
    for i in range(20):
        lens += 1
        q.copy_(torch.randn(2, 8, D, generator=gen(i)).bfloat16())
        k.copy_(torch.randn(2, 2, 1, D, generator=gen(100 + i)).bfloat16())
        v.copy_(torch.randn(2, 2, 1, D, generator=gen(200 + i)).bfloat16())
        graph.replay()
        want = se.step(q, k, v, lens)
        torch.cuda.synchronize()
        assert torch.equal(st.out, want) and torch.equal(st.block_idx, se.block_idx) and torch.equal(st.q_norm, se.q_norm)
    assert torch.equal(cache.bounds, other.bounds)
    if four_bits:
        assert torch.equal(cache.rows, other.rows) and torch.equal(cache.scales, other.scales)


def test_on_other_streams():
    """Calls go to the current stream, and two caches on two streams do not meet."""
    cases = [Case([350, 77], 8, 2, 32, "bf16", seed=82 + i) for i in range(2)]
    outs = []
    for c in cases:
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            c.append(c.lens)
            st = B.BlockDecodeState(c.dims, c.cache, 3, 10, 0, c.inv, 2048, True)
            lens = torch.tensor(c.lens, dtype=torch.int32, device="cuda")
            q = c.q.cuda()
            B.block_topk(c.dims, c.cache.blocks, q, st.cos_b, st.sin_b, st.q_rot, True, 3, 10, 0, lens, st.block_idx, st.block_count, ws=st.ws)
            B.sparse_attn_kv4(c.dims, c.cache, q, st.q_rot, st.block_idx, st.block_count, 3, 32, True, 10, 0, st.cos_win, st.sin_win, lens,
                              st.out, st.ws)
            y = torch.empty(2, 2, 350, D, dtype=torch.bfloat16, device="cuda")
            B.kv4_read(c.dims, c.cache, 350, lens, None, None, y)
            n = torch.empty(2, 8, 1, D, dtype=torch.bfloat16, device="cuda")
            B.qk_norm_rope(c.dims, q.reshape(2, 1, -1), None, 1, None, None, 1e-6, None, None, lens, q_norm=n)
            outs.append((st, lens, q, y, n))
    torch.cuda.synchronize()
    for c, (st, _, _, y, n) in zip(cases, outs):
        c.check_cache()
        sel = [[[j for j in st.block_idx[b, h].tolist() if j >= 0] for h in range(2)] for b in range(2)]
        check_attend(c, st.out.cpu(), st.q_rot.cpu(), st.cos_win.cpu().double(), st.sin_win.cpu().double(), sel, 32, True, 10, 0)
        assert torch.equal(y[0, 1].cpu().double(), c.seq(0, 1)[3])
        check(c.dims, c.q[:, None], None, 1, None, None, 1e-6, c.lens, None, {"q_norm": n.cpu()}, None)
