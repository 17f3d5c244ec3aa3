"""The operators on a key/value cache in 4 bits (a2ats_kv4_append, a2ats_kv4_read, a2ats_sparse_attn_kv4) against plain float64
forms, through the C ABI."""
import math
import os
import re

import pytest
import torch

import bench
from paper_2502_12665_amd import binding as B
from paper_2502_12665_amd import synth
from tests import kv4_ref as F
from tests import kv4_terms as K
from tests import kv_blocks_ref as R

pytestmark = pytest.mark.gpu
D = 128
U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}


def gen(seed):
    return torch.Generator().manual_seed(seed)


def up(n, m):
    return max(m, -(-n // m) * m)


class Case:
    """Sequences in host memory, and a cache on the GPU that appends fill."""

    def __init__(self, lens, heads, kv_heads, blk, dtype, page=0, seed=0, bounds=True, ctx=None):
        self.lens, self.blk, self.dtype, self.page = list(lens), blk, DT[dtype], page
        self.heads, self.kv_heads, self.G, self.batch = heads, kv_heads, heads // kv_heads, len(lens)
        self.ctx = max(max(lens), 1) if ctx is None else ctx
        self.stride = up(self.ctx, page or blk)
        g = gen(seed)
        # (groups of different sizes, so that their scales matter)
        size = lambda n: torch.exp2(torch.randint(-3, 2, (kv_heads, n, 4), generator=g).float()).repeat_interleave(32, -1)  # noqa: E731
        self.k = [(size(n) * torch.randn(kv_heads, n, D, generator=g)).to(self.dtype) for n in lens]
        self.v = [(size(n) * torch.randn(kv_heads, n, D, generator=g)).to(self.dtype) for n in lens]
        self.q = torch.randn(self.batch, heads, D, generator=g).to(self.dtype)
        self.dims = B.make_dims(self.batch, heads, kv_heads, D, 16, self.ctx, self.stride)
        table, n_pages = None, 0
        if page:
            slots = self.stride // page
            n_pages = self.batch * slots + 3
            table = torch.randperm(n_pages, generator=g)[: self.batch * slots].reshape(self.batch, slots).int().cuda()
        self.cache = B.Kv4Cache.empty(self.dims, blk, self.dtype, bounds, table, page, n_pages)
        self.cache.rows.fill_(0xA5)
        self.cache.scales.fill_(0xA5)
        if bounds:
            self.cache.bounds.fill_(-77.0)
        self.inv = synth.inv_freq(D, 500000.0)
        self.have = [0] * self.batch
        self.rounded = {}

    def append(self, upto, use_lens=True, n_new=None):
        """Bring sequence b to upto[b] tokens by one call."""
        m = [u - h for u, h in zip(upto, self.have)]
        n_new = max(max(m), 1) if n_new is None else n_new
        new = {x: torch.full((self.batch, self.kv_heads, n_new, D), 5.0, dtype=self.dtype) for x in "kv"}
        for b, (h, u) in enumerate(zip(self.have, upto)):
            new["k"][b, :, : u - h] = self.k[b][:, h:u]
            new["v"][b, :, : u - h] = self.v[b][:, h:u]
        lens = torch.tensor(upto, dtype=torch.int32, device="cuda")
        news = torch.tensor(m, dtype=torch.int32, device="cuda") if use_lens else None
        B.kv4_append(self.dims, self.cache, new["k"].cuda(), new["v"].cuda(), n_new, lens, news)
        self.have = list(upto)

    def piece(self, t, b, kv):
        """Part of a cache tensor that belongs to (b, kv): [slots, ...], pages put behind each other."""
        t = t.cpu()
        return t[b, kv] if not self.page else torch.cat([t[p, kv] for p in self.cache.page_table[b].tolist()])

    def seq(self, b, kv):
        """(rows, scales, keys, values) of the whole sequence."""
        if (b, kv) not in self.rounded:
            self.rounded[b, kv] = F.cached(self.k[b][kv], self.v[b][kv])
        return self.rounded[b, kv]

    def check_cache(self):
        """Everything that the cache holds is what the sequences so far say, and the rest is untouched."""
        torch.cuda.synchronize()
        for b in range(self.batch):
            n = self.have[b]
            for kv in range(self.kv_heads):
                rows, scales, _, _ = self.seq(b, kv)
                for got, want in ((self.cache.rows, rows), (self.cache.scales, scales)):
                    got = self.piece(got, b, kv)
                    assert torch.equal(got[:n], want[:n]), (b, kv)
                    assert (got[n:] == 0xA5).all()
                if self.cache.bounds is not None:
                    bd = self.piece(self.cache.bounds, b, kv).double()
                    touched = -(-n // self.blk)
                    assert torch.equal(bd[:touched], F.bounds(self.k[b][kv][:n], self.blk)), (b, kv)
                    assert (bd[touched:] == -77).all()


# ---------------------------------------------------------------------------------------------- append

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("blk, page", [(16, 0), (32, 64), (64, 64), (128, 0), (128, 256)])
def test_append_in_pieces(dtype, blk, page):
    """One token, a few, across block borders, more than a workgroup's rows, different numbers a sequence: after every call
    codes, scales and bounds are those of the whole sequences, and nothing else was written."""
    c = Case([400, 37, 1, 0, 261], 4, 2, blk, dtype, page, seed=blk + page)
    for s in [[1, 0, 0, 0, 5], [2, 1, 1, 0, 5], [blk - 1, 16, 1, 0, 6], [blk, 17, 1, 0, blk + 1], [blk + 1, 17, 1, 0, blk + 1],
              [min(400, blk + 130), 36, 1, 0, 200], [400, 37, 1, 0, 261]]:
        c.append(s)
        c.check_cache()


def test_append_all_at_once_and_padded():
    """Prefill of prompts of different lengths in one padded call: without new_lens a sequence's tokens are its first rows; and without
    any lengths."""
    c = Case([300, 1, 64, 0, 129], 7, 1, 32, "bf16", seed=3)
    c.append(c.lens, use_lens=False, n_new=300)
    c.check_cache()
    c = Case([515, 515], 8, 8, 64, "f32", seed=4, bounds=False)
    c.append([515, 515], use_lens=False)
    c.check_cache()
    c = Case([70, 70], 2, 2, 16, "bf16", seed=5)
    new = [torch.stack(t).cuda() for t in (c.k, c.v)]
    B.kv4_append(c.dims, c.cache, new[0], new[1], 70)
    c.have = [70, 70]
    c.check_cache()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rounding(dtype):
    """Numbers on the borders between codes and next to them, at scales from the least to the largest; zeros of both signs, groups of
    zeros, of tiny numbers, and of what is not finite or too large: codes and scales are equal."""
    dt = DT[dtype]
    mids = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float64)
    base = torch.cat([mids, F.E2M1]).repeat(2)[:30]
    groups = []
    for e in list(range(-103, -95)) + [-60, -1, 0, 1, 7, 60, 122, 123, 124, 125]:
        for lead in (6.0, 3.0 + 2.0 ** -7, 4.5, 5.999):
            for side in (0, 1, -1):
                x = (base * 2.0 ** e).float().to(dt)
                if side:
                    x = (x.double() * (1 + side * torch.finfo(dt).eps)).float().to(dt)
                x = torch.cat([x, torch.tensor([lead * 2.0 ** e, -0.0]).to(dt)])
                x[1::2] *= -1
                groups.append(x)
    for odd in (0.0, 2.0 ** -100, 2.0 ** -100 * (1 - 2.0 ** -8), 2.0 ** -126, 2.0 ** 127, 2.0 ** 127 * (1 - 2.0 ** -8), math.inf, -math.inf, math.nan, 3.3e38):
        x = torch.zeros(32, dtype=dt)
        x[5], x[9] = odd, -0.0
        groups.append(x)
        groups.append(x + torch.linspace(-1, 1, 32).to(dt))
    while len(groups) % 4:
        groups.append(torch.zeros(32, dtype=dt))
    x = torch.stack(groups).reshape(-1, D)
    n = x.shape[0]
    c = Case([n], 1, 1, 16, dtype, seed=6, bounds=False)
    c.k[0][0], c.v[0][0] = x, x.roll(1, 0)
    c.append([n])
    c.check_cache()


def test_tokens_written_again():
    """A sequence that goes back, also into a block: its tokens from there on are the new ones (bounds from a block's beginning on)."""
    c = Case([200], 2, 2, 32, "bf16", seed=8)
    c.append([200])
    other = Case([200], 2, 2, 32, "bf16", seed=9)
    for at in (64, 77, 90):                                # (77 and 90: codes and scales alone)
        c.k[0][:, at:], c.v[0][:, at:] = other.k[0][:, at:], other.v[0][:, at:]
        c.rounded.clear()
        c.have = [at]
        c.append([200])
        torch.cuda.synchronize()
        for kv in range(2):
            rows, scales, _, _ = c.seq(0, kv)
            assert torch.equal(c.piece(c.cache.rows, 0, kv)[:200], rows) and torch.equal(c.piece(c.cache.scales, 0, kv)[:200], scales)
            if at == 64:
                assert torch.equal(c.cache.bounds[0, kv].cpu().double()[:7], F.bounds(c.k[0][kv], 32))


def test_bounds_keep_what_is_not_finite():
    c = Case([50], 1, 1, 16, "f32", seed=10)
    c.k[0][0, 3, 7], c.k[0][0, 20, 9], c.k[0][0, 33, 11] = math.nan, math.inf, -math.inf
    for n in (1, 10, 33, 50):
        c.append([n])
    torch.cuda.synchronize()
    bd = c.cache.bounds[0, 0].cpu()[:4]
    want = F.bounds(c.k[0][0], 16)
    assert torch.isnan(bd[0, :, 7]).all() and torch.equal(torch.nan_to_num(bd.double(), nan=99.0), torch.nan_to_num(want, nan=99.0))


def test_bounds_of_bfloat16_of_both_signs_and_not_finite():
    """Zeros of both signs, the smallest and largest numbers, infinities; NaN of either sign, in a call or in one before, makes both bounds
    of its dimension NaN."""
    c = Case([48], 1, 1, 16, "bf16", seed=11)
    k = c.k[0][0]
    k[:, 0], k[:, 1] = k[:, 0].abs(), -k[:, 1].abs()
    k[3, 2], k[4, 2], k[5, 3], k[6, 4] = math.inf, -math.inf, -math.inf, math.inf
    k[:16, 5], k[16:, 5] = 0.0, -0.0
    k[:, 6] = torch.tensor([1, -1, 3, -3] * 12, dtype=torch.int16).view(torch.bfloat16) * 1.0
    k[7, 7], k[8, 7] = torch.finfo(torch.bfloat16).max, torch.finfo(torch.bfloat16).min
    k[2, 8], k[18, 9] = math.nan, torch.tensor([-1], dtype=torch.int16).view(torch.bfloat16)[0]
    for n in (9, 20, 48):
        c.append([n])
    torch.cuda.synchronize()
    bd, want = c.cache.bounds[0, 0].cpu()[:3].double(), F.bounds(k, 16)
    assert torch.isnan(bd[0, :, 8]).all() and torch.isnan(bd[1, :, 9]).all()
    assert torch.isnan(bd).sum() == 4 + 6                   # (dimension 6 has NaN with the sign, 0xffff and 0xfffd, beside the least numbers)
    assert torch.equal(torch.nan_to_num(bd, nan=99.0), torch.nan_to_num(want, nan=99.0))


# ---------------------------------------------------------------------------------------------- read back

@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("dtype, blk, page", [("bf16", 16, 0), ("f32", 32, 64), ("bf16", 128, 256)])
def test_read_back(out, dtype, blk, page):
    """All of the sequences, their last tokens, none; keys, values or both: code * scale, and later rows as they were."""
    c = Case([300, 37, 1, 0, 129], 4, 2, blk, dtype, page, seed=20 + blk, bounds=False)
    c.append(c.lens)
    lens = torch.tensor(c.lens, dtype=torch.int32, device="cuda")
    for n_rows, news in ((300, None), (65, None), (64, [64, 5, 1, 3, 0]), (1, None), (200, [-3, 100, 2, 0, 129])):
        m = [max(0, min(n_rows, x, n_rows if news is None else news[b])) for b, x in enumerate(c.lens)]
        nl = None if news is None else torch.tensor(news, dtype=torch.int32, device="cuda")
        for what in ("kv", "k", "v"):
            o = {x: torch.full((5, 2, n_rows, D), 9.0, dtype=DT[out], device="cuda") if x in what else None for x in "kv"}
            B.kv4_read(c.dims, c.cache, n_rows, lens, nl, o["k"], o["v"])
            torch.cuda.synchronize()
            for b in range(5):
                for kv in range(2):
                    for x in what:
                        got, want = o[x][b, kv].cpu().double(), c.seq(b, kv)[2 + "kv".index(x)]
                        assert torch.equal(got[: m[b]], want[c.lens[b] - m[b]:]), (n_rows, b, kv, x)
                        assert (got[m[b]:] == 9).all()


def test_read_back_of_what_is_not_finite():
    c = Case([40], 1, 1, 16, "f32", seed=22, bounds=False)
    c.k[0][0, 3, 40], c.v[0][0, 20, 127], c.v[0][0, 21] = math.nan, -math.inf, 0.0
    c.append([40])
    for dt in DT.values():
        k, v = (torch.zeros(1, 1, 40, D, dtype=dt, device="cuda") for _ in range(2))
        B.kv4_read(c.dims, c.cache, 40, None, None, k, v)
        k, v = k[0, 0].cpu(), v[0, 0].cpu()
        assert torch.isnan(k[3, 32:64]).all() and torch.isnan(k).sum() == 32
        assert torch.isnan(v[20, 96:]).all() and torch.isnan(v).sum() == 32 and (v[21] == 0).all()
        want = c.seq(0, 0)
        assert torch.equal(torch.nan_to_num(k.double()), torch.nan_to_num(want[2])) and torch.equal(torch.nan_to_num(v.double()), torch.nan_to_num(want[3]))


def test_read_keys_are_what_the_encoder_takes():
    """Keys of a cache in 4 bits, read back as float32, encoded against a codebook: the codes of those numbers."""
    c = Case([96, 96], 4, 2, 32, "bf16", seed=23, bounds=False)
    c.append(c.lens)
    keys = torch.empty(2, 2, 96, D, device="cuda")
    B.kv4_read(c.dims, c.cache, 96, None, None, keys, None)
    book = torch.randn(2, 16, 256, 8, generator=gen(24)).cuda()
    codes = torch.zeros(2, 2, 96, 16, dtype=torch.uint8, device="cuda")
    B.encode_keys(c.dims, keys, 96, 0, book, None, B.W_NONE, codes)
    k = torch.stack([torch.stack([c.seq(b, kv)[2] for kv in range(2)]) for b in range(2)]).unflatten(-1, (16, 8))
    dist = (k[..., None, :] - book.cpu().double()[None, :, None]).square().sum(-1)
    assert torch.equal(codes.cpu().long(), dist.argmin(-1))


# ---------------------------------------------------------------------------------------------- attention

def run_attend(c, sel, size, shared, window, n_sink, ws_fill=0xFF, q_rot=None, have=None):
    """sel [B, H] lists.  -> out, q_rot, tables."""
    H = c.kv_heads if shared else c.heads
    n_sel = max([len(x) for row in sel for x in row] + [1])
    idx = torch.full((c.batch, H, n_sel), -1, dtype=torch.int32)
    cnt = torch.zeros(c.batch, H, dtype=torch.int32)
    for b in range(c.batch):
        for h in range(H):
            idx[b, h, : len(sel[b][h])] = torch.tensor(sel[b][h], dtype=torch.int32)
            cnt[b, h] = len(sel[b][h])
    cos_b, sin_b, cos_w, sin_w = B.rope_tables(D, c.inv, 2048, window, "cuda")
    if q_rot is None:
        q_rot = R.rotate(c.q.double(), cos_b.cpu().double(), sin_b.cpu().double()).float()
    ws = torch.full((max(16, B.workspace_bytes(c.dims, B.OP_ATTN_KV4, n_sel * size, window)),), ws_fill, dtype=torch.uint8, device="cuda")
    out = torch.full((c.batch, c.heads, D), 3.0, dtype=c.dtype, device="cuda")
    sl = torch.tensor(c.have if have is None else have, dtype=torch.int32, device="cuda")
    B.sparse_attn_kv4(c.dims, c.cache, c.q.cuda(), q_rot.cuda(), idx.cuda(), cnt.cuda(), n_sel, size, shared, window, n_sink,
                      cos_w, sin_w, sl, out, ws)
    torch.cuda.synchronize()
    return out.cpu(), q_rot, cos_w.cpu().double(), sin_w.cpu().double()


def check_attend(c, got, q_rot, cos_w, sin_w, sel, size, shared, window, n_sink):
    half_step = HALF[c.dtype]
    for b in range(c.batch):
        n = c.have[b]
        lo, hi = R.candidates(n, window, n_sink)
        for h in range(c.heads):
            kv = h // c.G
            _, _, k, v = c.seq(b, kv)
            picked = sel[b][kv if shared else h]
            pos = [j for j in picked if lo <= j < hi] if size == 1 else R.tokens_of(picked, n, c.blk, window, n_sink)
            want, off = R.attend(c.q[b, h].double(), q_rot[b, h].double(), k, v, n, pos, window, n_sink, cos_w, sin_w)
            err = (got[b, h].double() - want).abs()
            tol = off * (1 + half_step) + half_step * want.abs()
            assert (err <= tol).all(), (b, h, float((err - tol).max()), float(err.max()))


def draw_sel(c, size, shared, n_sel, window, n_sink, seed):
    g = gen(seed)
    H = c.kv_heads if shared else c.heads
    sel = []
    for b in range(c.batch):
        lo, hi = R.candidates(c.have[b], window, n_sink)
        units = list(range(lo // size, (hi - 1) // size + 1)) if hi > lo else []
        sel.append([[units[i] for i in torch.randperm(len(units), generator=g).tolist()[:n_sel]] for _ in range(H)])   # (in any order)
    return sel


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("blk, page, unit, window, n_sink, n_sel", [
    (16, 0, 1, 64, 0, 100), (32, 64, 1, 5, 3, 40), (64, 0, 64, 0, 0, 3), (128, 128, 128, 20, 40, 2), (16, 32, 16, 300, 1, 7),
    (32, 0, 1, 1, 700, 10)])
@pytest.mark.parametrize("shared", [False, True])
def test_attention(dtype, blk, page, unit, window, n_sink, n_sel, shared):
    """Lengths around a block, windows from none to more than the sequence, sinks past the end."""
    c = Case([0, 1, blk - 1, blk, blk + 1, 530], 6, 2, blk, dtype, page, seed=blk + n_sel, bounds=False)
    c.append(c.lens)
    sel = draw_sel(c, unit, shared, n_sel, window, n_sink, 40)
    got = run_attend(c, sel, unit, shared, window, n_sink)
    check_attend(c, *got, sel, unit, shared, window, n_sink)


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 7, 8])
def test_attention_of_every_group(G, shared):
    c = Case([901, 300], 2 * G, 2, 32, "bf16" if G % 3 else "f32", seed=50 + G, bounds=False)
    c.append(c.lens)
    for unit, n_sel in ((1, 333), (32, 11)):
        sel = draw_sel(c, unit, shared, n_sel, 48, 2, 51)
        got = run_attend(c, sel, unit, shared, 48, 2)
        check_attend(c, *got, sel, unit, shared, 48, 2)


@pytest.mark.parametrize("batch, heads, kv_heads, n, n_sel, shared", [
    (1, 4, 1, 5000, 4096, False), (1, 8, 1, 5000, 4096, True), (40, 8, 1, 700, 300, False), (70, 8, 8, 600, 256, True)])
def test_attention_shared_out_or_not(batch, heads, kv_heads, n, n_sel, shared):
    """Few heads of many rows (several workgroups a head), and many heads of few."""
    c = Case([n] * min(batch, 2) + [17] * (batch - min(batch, 2)), heads, kv_heads, 16, "f32", seed=60, bounds=False)
    c.append(c.lens)
    sel = draw_sel(c, 1, shared, n_sel, 100, 4, 61)
    got = run_attend(c, sel, 1, shared, 100, 4)
    check_attend(c, *got, sel, 1, shared, 100, 4)
    again = run_attend(c, sel, 1, shared, 100, 4, ws_fill=0x00)
    assert torch.equal(got[0], again[0])                    # the workspace's contents do not matter, nor the run


@pytest.mark.parametrize("shared", [False, True])
def test_graphs_with_one_workspace(shared):
    """Two captured calls of several workgroups a head that have one workspace, replayed in turn with other calls in it between."""
    cases = [Case([900], 4, 1, 16, dtype, seed=63 + i, bounds=False) for i, dtype in enumerate(("f32", "bf16"))]
    graphs, ws, side = [], torch.empty(1 << 20, dtype=torch.uint8, device="cuda"), torch.cuda.Stream()
    for c in cases:
        c.append(c.lens)
        sel = draw_sel(c, 1, shared, 800, 40, 2, 65)
        want, q_rot, cos_w, sin_w = run_attend(c, sel, 1, shared, 40, 2)           # (the kernels are loaded before the capture)
        need = B.workspace_bytes(c.dims, B.OP_ATTN_KV4, 800, 40)
        assert 4 * 130 * 4 * 2 <= need <= ws.numel()                               # (two parts at least)
        args = [c.q.cuda(), q_rot.cuda(), torch.tensor(sel, dtype=torch.int32, device="cuda"),
                torch.full((1, 1 if shared else 4), 800, dtype=torch.int32, device="cuda"), 800, 1, shared, 40, 2, cos_w.float().cuda(),
                sin_w.float().cuda(), torch.tensor([900], dtype=torch.int32, device="cuda")]
        out = torch.empty(1, 4, D, dtype=c.dtype, device="cuda")
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            B.sparse_attn_kv4(c.dims, c.cache, *args, out, ws)
        graphs.append((graph, out, want, args))
    for _ in range(4):
        for graph, out, want, _ in graphs:
            out.fill_(9.0)
            ws.fill_(0xFF)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out.cpu(), want)


@pytest.mark.parametrize("shared, heads", [(False, 6), (True, 6), (True, 16)])
def test_what_is_not_attended(shared, heads):
    """Indices outside of the candidates, below zero and beyond the sequence, and counts outside of their range: left out; nothing attended: zeros, also for
    a query that is not finite."""
    c = Case([100, 100, 64], heads, 2, 16, "f32", seed=70, bounds=False, ctx=200)
    c.append([100, 100, 0])
    H = 2 if shared else heads
    sel = [[[3, 99, 500, -1, 8, 95, 1 << 30, 0, 111]] * H, [[98, 2000000000, 1, -5]] * H, [[0, 5]] * H]
    got = run_attend(c, sel, 1, shared, 6, 2)               # candidates [2, 94)
    check_attend(c, *got, sel, 1, shared, 6, 2)
    assert (got[0][2] == 0).all()
    c.q[0] = math.nan
    c.q[1] = math.inf
    out = run_attend(c, [[[-1, 100]] * H] * 3, 1, shared, 0, 0)[0]
    assert (out == 0).all()
    idx = torch.tensor([4, 5], dtype=torch.int32, device="cuda").expand(3, H, 2).contiguous()
    cos_b, sin_b, cos_w, sin_w = B.rope_tables(D, c.inv, 2048, 4, "cuda")
    for count in (-3, 7):
        o = torch.full((3, heads, D), 3.0, device="cuda")
        q = torch.randn(3, heads, D, generator=gen(71)).cuda()
        ws = torch.empty(max(16, B.workspace_bytes(c.dims, B.OP_ATTN_KV4, 2, 0)), dtype=torch.uint8, device="cuda")
        B.sparse_attn_kv4(c.dims, c.cache, q, q, idx, torch.full((3, H), count, dtype=torch.int32, device="cuda"), 2, 1, shared, 0, 0, None, None,
                          torch.tensor([100, 100, 0], dtype=torch.int32, device="cuda"), o, ws)
        assert (o[:2] != 0).any() == (count > 0) and (o[2] == 0).all()


@pytest.mark.parametrize("shared, heads", [(False, 4), (True, 4), (True, 14)])
@pytest.mark.parametrize("window", [0, 64])
def test_what_is_not_finite(shared, heads, window):
    """A key, value or query that is not finite is seen by the heads that attend it and by no others; of a value, in its group."""
    c = Case([128, 128, 128], heads, 2, 32, "f32", seed=72, bounds=False)
    c.k[0][0, 100, 5] = math.nan
    c.v[1][1, 90, 70] = math.inf
    c.append(c.lens)
    c.q[2, 0, 3] = math.inf
    c.q[2, heads - 1, 127] = math.nan
    H = 2 if shared else heads
    near = [] if window else [100, 90]
    sel = [[near + [5, 17, 40]] * H] * 3
    got = run_attend(c, sel, 1, shared, window, 0)[0]
    G = heads // 2
    bad = torch.isnan(got)
    assert bad[0, :G].all() and not bad[0, G:].any()
    assert bad[1, G:, 64:96].all() and bad[1].sum() == G * 32
    assert bad[2, 0].all() and bad[2, -1].all() and not bad[2, 1:-1].any()
    free = run_attend(c, [[[5, 17, 40]] * H] * 3, 1, shared, 0, 0)[0]   # rows that nobody selects do not matter
    assert torch.isfinite(free[:2]).all()


@pytest.mark.parametrize("G, shared", [(1, False), (4, False), (3, True), (4, True), (6, True), (8, True)])
@pytest.mark.parametrize("window", [0, 12])
def test_low_bits_of_queries_and_keys(G, shared, window):
    """Keys of four elements that are not zero: few roundings, which are counted."""
    batch, Hkv, n, rows = 4, 2, 64, 12
    g = gen(80 + G)
    c = Case([n] * batch, Hkv * G, Hkv, 16, "f32", seed=81, bounds=False)
    for b in range(batch):
        keep = torch.rand(Hkv, n, D, generator=g).argsort(-1).argsort(-1) < 4
        c.k[b] = torch.randn(Hkv, n, D, generator=g) * keep * 20
        c.v[b] = torch.randn(Hkv, n, D, generator=g)
    c.append(c.lens)
    H = Hkv if shared else c.heads
    sel = [[[] if window else torch.randperm(n, generator=g)[:rows].tolist() for _ in range(H)] for _ in range(batch)]
    q_rot = torch.randn(batch, c.heads, D, generator=g)
    got, _, cos, sin = run_attend(c, sel, 1, shared, window, 0, q_rot=q_rot)
    for b in range(batch):
        for h in range(c.heads):
            at = torch.tensor(list(range(n - rows, n)) if window else sel[b][h // G if shared else h])
            k, v = (t[at] for t in c.seq(b, h // G)[2:])
            q = (c.q if window else q_rot)[b, h].double()
            size, small = k.abs(), 0.0
            if window:
                cs, sn = cos[n - 1 - at], sin[n - 1 - at]
                k1, k2 = k[:, :64], k[:, 64:]
                size = torch.cat([k1.abs() * cs.abs() + k2.abs() * sn.abs(), k2.abs() * cs.abs() + k1.abs() * sn.abs()], -1)
                # float16 terms of a key, relative to its row's largest scale (at most a third of its largest element): 2^-25 of it each
                small = 2.0 ** -25 * k.abs().amax(-1) / 3 * q.abs().sum()
                # ... and of a query, relative to the least power of two above it: 2^-33
                small = small + 2.0 ** -32 * q.abs().max() * size.sum(-1)
                k = torch.cat([k1 * cs + k2 * sn, k2 * cs - k1 * sn], -1)
            logit = k @ q / math.sqrt(D)
            p = logit.softmax(0)
            # In steps of u of sum |q| |k|: the query's factor and its rounding (2), a turned key's products and sum (3), the float16 terms
            # (2 for the key, 2 for the query), 8 elements' terms added by the matrix cores, truncated each (32), the terms' sum (3),
            # the scale (1): 45 < 48.
            d = ((48 * U * (size @ q.abs()) + small) / math.sqrt(D)).max() + (3 * float(logit.abs().max()) + 12 + 6 * rows) * U
            want, tol = p @ v, 2 * d * (p @ v.abs()) + U * (p @ v).abs()
            err = (got[b, h].double() - want).abs()
            assert (err <= tol).all(), (b, h, float((err / tol).max()))


@pytest.mark.parametrize("what, G, shared", K.ALL)
def test_low_terms_of_queries_and_turned_keys(what, G, shared):
    """Inputs of tests/kv4_terms.py, in which a term that is left out shows."""
    t = K.Terms(what, G, shared, seed=G)
    c = Case([K.N] * K.B, t.heads, K.HKV, 16, "f32", seed=82, bounds=False)
    c.k, c.v, c.q = list(t.k), list(t.v), t.q
    c.append(c.lens)
    got, _, cos, sin = run_attend(c, t.sel, 1, shared, t.window, 0, q_rot=t.q)
    for b in range(K.B):
        for h in range(t.heads):
            want, tol = t.want(b, h, cos, sin)
            err = (got[b, h].double() - want).abs()
            assert (err <= tol).all(), (b, h, float((err / tol.clamp(min=1e-30)).max()))


@pytest.mark.parametrize("G, shared", [(1, False), (4, True), (5, True), (8, True)])
@pytest.mark.parametrize("window", [0, 2])
def test_weights_have_24_bits(G, shared, window):
    """Two rows, values of 1 and 0: the output is a softmax weight.  Logits of one element: the key is a number of 2 bits and the query's
    product with it is exact in each term."""
    batch, n = 24, 16
    g = gen(90 + G)
    c = Case([n] * batch, G, 1, 16, "f32", seed=91, bounds=False)
    for b in range(batch):
        c.k[b], c.v[b] = torch.zeros(1, n, D), torch.zeros(1, n, D)
        c.k[b][0, n - 2:, 63] = torch.tensor([1.0, -1.0])
        c.v[b][0, n - 2] = 1.0
    c.append(c.lens)
    c.q = torch.zeros(batch, G, D)
    c.q[..., 63] = 8 * torch.rand(batch, G, generator=g) - 4
    c.inv = torch.zeros(64, dtype=torch.float64)            # (no rotation: window rows are not turned)
    got = run_attend(c, [[[] if window else [n - 2, n - 1]] * (1 if shared else G)] * batch, 1, shared, window, 0, q_rot=c.q)[0].double()
    x = 2 * c.q[..., 63].double() / math.sqrt(D)
    want = torch.sigmoid(x)[..., None]
    # The logits' difference, |x| <= 0.71, times log2 e: three roundings of each (its factor, its rounding, the terms' sum) and that of the
    # difference: 7 u |x|; an exponential each (2 u), their sum, a weight's terms (truncated additions: 6 u), joining waves (4 u), the division:
    # below 24 u.  A weight of 16 bits is off by up to 2^-16 = 256 u.
    assert ((got - want).abs() <= 24 * U * want).all(), float(((got - want).abs() / want).max() / U)


@pytest.mark.parametrize("G, shared", [(4, False), (4, True), (7, True)])
@pytest.mark.parametrize("window", [0, 8])
def test_keys_and_values_of_any_size(G, shared, window):
    """Scales of 2^90 and 2^-90 in one row's groups, queries that make ordinary logits of them, and tiny values."""
    batch, n, rows = 3, 32, 8
    g = gen(95)
    c = Case([n] * batch, G, 1, 16, "f32", seed=96, bounds=False)
    c.inv = torch.zeros(64, dtype=torch.float64)
    scale = torch.tensor([2.0 ** 90, 2.0 ** -90, 1.0, 2.0 ** 30]).repeat_interleave(32)
    for b in range(batch):
        keep = torch.zeros(D)
        keep[[3, 40, 70, 100]] = 1.0
        c.k[b] = torch.randint(-6, 7, (1, n, D), generator=g) * keep * scale
        c.v[b] = torch.randint(-6, 7, (1, n, D), generator=g) * torch.tensor([2.0 ** -90, 2.0 ** 90, 1.0, 2.0 ** -30]).repeat_interleave(32)
    c.append(c.lens)
    c.q = torch.zeros(batch, G, D)
    c.q[..., 3] = 2.0 ** -90 * torch.randn(batch, G, generator=g)
    if not window:                                          # (turned keys keep 2^-26 of the row's largest element)
        c.q[..., 40], c.q[..., 70], c.q[..., 100] = (s * torch.randn(batch, G, generator=g) for s in (2.0 ** 90, 1.0, 2.0 ** -30))
    sel = [[[] if window else torch.randperm(n, generator=g)[:rows].tolist() for _ in range(1 if shared else G)] for _ in range(batch)]
    got = run_attend(c, sel, 1, shared, window, 0, q_rot=c.q)[0].double()
    for b in range(batch):
        for h in range(G):
            at = list(range(n - window, n)) if window else sel[b][0 if shared else h]
            k, v = (t[at] for t in c.seq(b, 0)[2:])
            q = c.q[b, h].double()
            logit = k @ q / math.sqrt(D)
            p = logit.softmax(0)
            d = 48 * U * float((k.abs() @ q.abs()).max()) / math.sqrt(D) + (3 * float(logit.abs().max()) + 12 + 6 * rows) * U
            assert ((got[b, h] - p @ v).abs() <= (2 * d + U) * (p @ v.abs())).all(), (b, h)


@pytest.mark.parametrize("G, shared", [(1, False), (3, True), (7, True)])
@pytest.mark.parametrize("small, large", [(2.0 ** -97, 2.0 ** 122), (2.0 ** 122, 2.0 ** -97)])
def test_window_of_factors_far_apart(G, shared, small, large):
    """Queries and window keys whose factors are at either end of float32, with logits between: 2^25 and a quarter of it, so that the
    output is the first key's value."""
    c = Case([8], G, 1, 16, "f32", seed=99, bounds=False)
    c.inv = torch.zeros(64, dtype=torch.float64)
    c.k[0] = torch.full((1, 8, D), 0.25 * large)
    c.k[0][:, 5] = large
    c.append(c.lens)
    c.q = torch.full((1, G, D), small)
    got = run_attend(c, [[[] for _ in range(1 if shared else G)]], 1, shared, 8, 0, q_rot=c.q)[0]
    want = c.seq(0, 0)[3][5]
    assert torch.equal(got[0].double(), want.expand(G, D))


def test_lengths_outside_of_their_range_are_limited():
    """seq_lens below 0 and above ctx_len, new_lens below 0, above n_new and above the sequence's length: the nearest that can be."""
    c = Case([96, 96, 96, 96], 4, 2, 32, "bf16", seed=97)
    want = Case([96, 96, 96, 96], 4, 2, 32, "bf16", seed=97)
    new = [torch.stack(t).cuda() for t in (c.k, c.v)]
    odd = [[1000, 96, -7, 10], [2000, -3, 50, 96]], [[96, 96, 0, 10], [96, 0, 0, 10]]
    back = []
    for x, (sl, nl) in zip((c, want), odd):
        sl, nl = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in (sl, nl))
        B.kv4_append(x.dims, x.cache, *new, 96, sl, nl)
        o = [torch.zeros(4, 2, 96, D, device="cuda") for _ in range(2)]
        B.kv4_read(x.dims, x.cache, 96, sl, nl, *o)
        back.append(o)
    torch.cuda.synchronize()
    for x in ("rows", "scales", "bounds"):
        assert torch.equal(getattr(c.cache, x), getattr(want.cache, x)), x
    assert all(torch.equal(a, b) for a, b in zip(*back))
    c.append([96] * 4)
    outs = [run_attend(c, [[[0, 2]] * 4] * 4, 32, False, 7, 1, have=h)[0] for h in ([1000, 96, -7, 96], [96, 96, 0, 96])]
    assert torch.equal(*outs) and (outs[0][2] == 0).all()


def test_a_pool_of_more_than_4_gib():
    """Pages behind the first 2^32 bytes of a pool: append, read back, select and attend there."""
    page, blk, Hkv = 64, 32, 8
    n_pages = (1 << 32) // (Hkv * page * D) + 300
    n = 300
    slots = up(n, page) // page
    dims = B.make_dims(1, 8, Hkv, D, 16, n, up(n, page))
    table = torch.arange(n_pages - 1, n_pages - 1 - 2 * slots, -2, dtype=torch.int32).reshape(1, slots).cuda()
    c = Case([n], 8, Hkv, blk, "bf16", seed=98)
    c.page, c.dims, c.cache = page, dims, B.Kv4Cache.empty(dims, blk, torch.bfloat16, True, table, page, n_pages)
    c.append([n], use_lens=False)
    k, v = (torch.zeros(1, Hkv, n, D, device="cuda") for _ in range(2))
    B.kv4_read(dims, c.cache, n, None, None, k, v)
    for kv in range(Hkv):
        assert torch.equal(k[0, kv].cpu().double(), c.seq(0, kv)[2]) and torch.equal(v[0, kv].cpu().double(), c.seq(0, kv)[3])
    sel = draw_sel(c, blk, False, 3, 20, 2, 99)
    got = run_attend(c, sel, blk, False, 20, 2)
    check_attend(c, *got, sel, blk, False, 20, 2)


# ---------------------------------------------------------------------------------------------- steps

@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("ctx", [1024, 1003])
def test_steps_of_the_benchmark(shared, ctx):
    """Through the last block twice and a half: the cache holds the sequence up to each step's token, and its selection and output are those
    of that sequence."""
    wl = synth.WORKLOADS["c1_tiny"].replace(batch=2, ctx_len=ctx, top_k=96, window=40)
    run = bench.BlockCacheSteps(torch, B, synth, wl, "e2m1", shared)
    x = synth.make_decode_inputs(wl, device="cuda")
    k, v, q = (x[c].cpu() for c in ("k", "v", "q"))
    st, c = run.state, run.cache
    cos_w, sin_w = st.cos_win.cpu().double(), st.sin_win.cpu().double()
    for i in range(run.tokens * 5 // 2):
        out = run.step(i)
        n = run.first + i % run.tokens + 1
        if i % run.tokens not in (0, 1, 9, run.tokens - 1):
            continue
        torch.cuda.synchronize()
        for b in range(2):
            rows, scales, kk, vv = F.cached(k[b, 0, :n], v[b, 0, :n])
            assert torch.equal(c.rows[b, 0, :n].cpu(), rows) and torch.equal(c.scales[b, 0, :n].cpu(), scales)
            bd = F.bounds(k[b, 0, :n], 16)
            assert torch.equal(c.bounds[b, 0].cpu().double()[: -(-n // 16)], bd)
            q_rot = st.q_rot[b].cpu().double()
            picked = R.select(q_rot, bd, n, 16, 40, wl.n_sink, 6, shared)
            for h in range(4):
                blocks = picked[0 if shared else h][0]
                assert st.block_idx[b, 0 if shared else h].tolist() == blocks
                want, off = R.attend(q[b, h].double(), q_rot[h], kk, vv, n, R.tokens_of(blocks, n, 16, 40, wl.n_sink), 40, wl.n_sink, cos_w, sin_w)
                half = HALF[st.out.dtype]
                assert ((out[b, h].cpu().double() - want).abs() <= off * (1 + half) + half * want.abs()).all(), (i, b, h)


def test_the_readme_program():
    """README.md's code blocks as they stand, behind each other: after 20 tokens of a model with norms the cache holds the prompt's normalised
    keys, and the last output is the attention of what was selected."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = "\n".join(re.findall(r"```python\n(.*?)```", open(os.path.join(root, "README.md")).read(), re.S))
    at = code.index("# or blocks selected")
    env = {}
    exec(code[:at], env)
    wl, x = env["wl"], env["x"]
    N, w, G = wl.ctx_len, wl.window, wl.n_q_heads // wl.n_kv_heads
    g = gen(2)
    new = [[torch.randn(1, n, D, generator=g).bfloat16() for n in (wl.n_q_heads, wl.n_kv_heads, wl.n_kv_heads)] for _ in range(20)]
    env["tokens"] = [(q.cuda(), k.unsqueeze(2).cuda(), v.unsqueeze(2).cuda()) for q, k, v in new]
    exec(code[at:], env)
    torch.cuda.synchronize()
    n, bs, four = N + 20, env["bs4"], env["four"]
    assert env["lens4"].tolist() == [n]
    cos_w, sin_w = bs.cos_win.cpu().double(), bs.sin_win.cpu().double()
    want_q = F.norm(new[-1][0].double(), env["q_weight"].cpu(), 1e-6)
    assert ((bs.q_norm.cpu().double() - want_q).abs() <= F.half_step(want_q, torch.bfloat16) + 2 * F.NORM_ROUNDINGS * U * want_q.abs()).all()
    back = [torch.empty(1, wl.n_kv_heads, n, D, device="cuda") for _ in range(2)]
    B.kv4_read(env["grown"], four, n, env["lens4"], None, *back)
    assert all(torch.equal(t[:, :, 20:], env[name]) for t, name in zip(back, ("k_back", "v_back")))
    for h in (0, wl.n_q_heads - 1):
        kv = h // G
        rows, scales, k, v = F.cached(env["k_norm"][0, kv].cpu(), x["v"][0, kv].cpu())
        assert torch.equal(four.rows[0, kv, :N].cpu(), rows) and torch.equal(four.scales[0, kv, :N].cpu(), scales)
        kk, vv = (t[0, kv].cpu().double() for t in back)
        assert torch.equal(kk[:N], k) and torch.equal(vv[:N], v)
        blocks = bs.block_idx[0, h].tolist()
        assert len(blocks) == wl.top_k // 16 and min(blocks) >= 0
        want, off = R.attend(bs.q_norm[0, h].cpu().double(), bs.q_rot[0, h].cpu().double(), kk, vv, n, R.tokens_of(blocks, n, 16, w, 0), w, 0,
                             cos_w, sin_w)
        err = (env["out4"][0, h].cpu().double() - want).abs()
        assert (err <= off * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs()).all(), (h, float(err.max()))
