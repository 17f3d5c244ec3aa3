"""Operators around a key/value cache held in 4 bits, as cases that can be timed and compared.

Five kinds of call:

  norm    queries and keys of new tokens are normalised head by head, and rotated by their positions, in one pass
  write   new tokens enter a cache held in 4 bits (e2m1 numbers, a power of two for each 32 of them), with the bounds of the
          blocks' keys, and are read back as the values that they now stand for
  read    a prompt's cached keys and values are read back
  attend  one query token attends the sinks, the selected tokens or blocks, and the recent window of such a cache
  step    a decode step of one layer: append the current token, select blocks, attend

With `own` false, run() computes them from elementary torch operations; with `own` true it makes the library's calls.
exact() computes the same in float64 from the definitions, apart from both.

A cached row is 128 bytes: 64 of the key's codes, byte i with dimensions 2 i (low half) and 2 i + 1, then 64 of the value's, byte
4 n + g with dimensions 32 g + 2 n and 32 g + 2 n + 1.  Its scales are 8 bytes, exponents + 127: the key's four groups of 32
dimensions, then the value's.
"""
from __future__ import annotations

import math

import torch

own = False

D = 128
HALF = D // 2
GROUP = 32
DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
TINY = 2.0 ** -100   # a group whose largest magnitude is below this is stored as zeros
EPS = 1e-6


def _case(name, kind, batch, heads, kv_heads, ctx, **opts):
    case = {"name": name, "kind": kind, "batch": batch, "heads": heads, "kv_heads": kv_heads, "ctx": ctx, "block": 32,
            "dtype": "bf16", "page": 0, "ragged": False, "new": 1, "bounds": True, "window": 64, "sink": 0, "n_sel": 0,
            "unit": "blocks", "shared": False, "rotate": True, "packed": True}
    case.update(opts)
    return case


def listed():
    return [
        # One decode step's queries and keys of 16 users, for the cache and the selection: launch and latency.
        _case("norm_token_b16", "norm", 16, 32, 8, 8192, ragged=True, rotate=False),
        # A prompt of 32768 tokens out of one packed projection, the benchmark's 8B shape: a stream through the card.
        _case("norm_prefill_32k", "norm", 1, 32, 8, 32768, new=32768),
        # A chunk of up to 1021 tokens of four sequences wherever they end, float32, projections of their own.
        _case("norm_chunk_f32", "norm", 4, 28, 4, 16384, new=1021, dtype="f32", ragged=True, packed=False),
        # One decode step's new token for 16 users: launch and latency.
        _case("write_token_b16", "write", 16, 32, 8, 8192, ragged=True),
        # Prefill of one prompt of 32768 tokens.
        _case("write_prefill_32k", "write", 1, 32, 8, 32768, new=32768),
        # A chunk of up to 4099 tokens appended to four sequences wherever they end, float32, in pages.
        _case("write_chunk_f32_paged", "write", 4, 28, 4, 16384, block=64, new=4099, dtype="f32", page=128, ragged=True),
        # A prompt of 65536 tokens read back, for the attention of its next chunk or for the key encoder.
        _case("read_prompt_64k", "read", 1, 28, 4, 65536, new=65536),
        # The smallest attention: one KV head, 128 tokens and a window of 64, float32.
        _case("attend_tiny_f32", "attend", 1, 4, 1, 4096, block=16, n_sel=128, unit="tokens", dtype="f32"),
        # The tokens that the code scores select, of four sequences of 131072: rows scattered over the cache.
        _case("attend_tokens_b4_128k", "attend", 4, 32, 8, 131072, n_sel=2048, unit="tokens", window=256),
        # The most rows: 32 sequences x 28 heads x 2048 tokens.
        _case("attend_tokens_b32_64k", "attend", 32, 28, 4, 65536, n_sel=2048, unit="tokens", window=128),
        # One selection of blocks a KV head, in pages, sequences of their own lengths, with sinks.
        _case("attend_shared_b16_32k_paged", "attend", 16, 32, 8, 32768, n_sel=32, window=128, sink=4, shared=True, ragged=True, page=64),
        # A whole step of four long conversations of an odd length.
        _case("step_b4_128k", "step", 4, 32, 8, 131001, n_sel=64, window=256, sink=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of the same ranges: 1 to 32 sequences, 64 to 131072 tokens, 1 to 8 query heads a KV head."""
    while True:
        kind = rng.choice(["norm", "write", "read", "attend", "attend", "step"])
        kv_heads = rng.choice([1, 2, 4, 8])
        heads = kv_heads * rng.randint(1, 8)
        batch, ctx, block = _log(rng, 1, 32), _log(rng, 64, 131072), rng.choice([16, 32, 64, 128])
        page = block * rng.choice([1, 2, 4]) if rng.random() < 0.4 else 0
        c = _case("", kind, batch, heads, kv_heads, ctx, block=block, page=page, dtype=rng.choice(["bf16", "bf16", "f32"]),
                  ragged=rng.random() < 0.4, window=_log(rng, 1, 512) - 1, sink=rng.choice([0, 0, 1, 4, 33]),
                  shared=rng.random() < 0.4, rotate=rng.random() < 0.7, packed=rng.random() < 0.6)
        del c["name"]
        wide = 2 if c["dtype"] == "f32" else 1
        if kind in ("norm", "write", "read"):
            c["new"] = _log(rng, 1, ctx)
            c["bounds"] = kind == "write" and rng.random() < 0.7
        if kind == "step":
            c["n_sel"] = max(1, min(1024, _log(rng, 8, 4096) // block))
        if kind == "attend":
            c["unit"] = rng.choice(["tokens", "blocks"])
            n = _log(rng, 8, 4096)
            c["n_sel"] = n if c["unit"] == "tokens" else max(1, n // block)
        if kind == "norm" and batch * (heads + kv_heads) * c["new"] * wide > 40 * 32768:
            continue
        if kind != "norm" and (batch * kv_heads * ctx > 8 << 20 or batch * kv_heads * c["new"] * wide > 32768 * 8):
            continue
        rows = c["n_sel"] * (block if c["unit"] == "blocks" else 1) + c["window"]
        if kind in ("attend", "step") and batch * heads * rows > 32 * 28 * 2176:
            continue
        return c


# ---------------------------------------------------------------------------------------------- inputs

def _lengths(case, g):
    """Tokens of each sequence, the new ones included; None: all have `ctx`."""
    if not case["ragged"]:
        return None
    n = torch.randint(max(1, case["ctx"] // 3), case["ctx"] + 1, (case["batch"],), generator=g, device=DEV, dtype=torch.int32)
    n[0] = case["ctx"]
    return n


def _normal(shape, dtype, g):
    return torch.randn(shape, generator=g, device=DEV).to(dtype)


def _codes(x):
    """e2m1 codes (sign in bit 3) and scale bytes of rows x [..., 128], 32 bits."""
    x = x.float().unflatten(-1, (D // GROUP, GROUP))
    a = x.abs().amax(-1)
    some = a >= TINY
    m, e = torch.frexp(torch.where(some, a, 1.0))
    e = e - 3 + (m > 0.75).to(e.dtype)                     # 6 = 0.75 * 2^3
    y = (x * torch.exp2(-e.float())[..., None]).abs()
    code = (y > 0.25).to(torch.uint8)
    code += y >= 0.75                                      # a tie goes to the even code
    code += y > 1.25
    code += y >= 1.75
    code += y > 2.5
    code += y >= 3.5
    code += y > 5.0
    code |= x.signbit().to(torch.uint8) << 3
    code = torch.where(some[..., None], code, 0)
    return code.flatten(-2), torch.where(some, e + 127, 0).to(torch.uint8)


def _cached(x_k, x_v):
    """Rows [..., 128] and scales [..., 8] of a cache, both bytes, that hold keys and values."""
    (ck, sk), (cv, sv) = _codes(x_k), _codes(x_v)
    k = ck[..., 0::2] | ck[..., 1::2] << 4
    v = (cv[..., 0::2] | cv[..., 1::2] << 4).unflatten(-1, (4, 16)).transpose(-1, -2).flatten(-2)
    return torch.cat([k, v], -1), torch.cat([sk, sv], -1)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 23)
    B, Hq, Hkv, blk, page = case["batch"], case["heads"], case["kv_heads"], case["block"], case["page"]
    dt, kind, new, w = DTYPES[case["dtype"]], case["kind"], case["new"], case["window"]
    unit = page or blk
    slots = -(-case["ctx"] // unit)            # pages (or blocks) of a sequence
    stride = slots * unit
    s = {"case": dict(case), "stride": stride, "seq_lens": _lengths(case, g), "new_lens": None}
    if case["ragged"] and new > 1:
        s["new_lens"] = torch.randint(0, new + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
        s["new_lens"][0] = new
    inv = torch.exp(-torch.arange(HALF, dtype=torch.float64, device=DEV) / HALF * math.log(500000.0))
    if kind == "norm":
        s["k_weight"] = 1 + 0.2 * torch.randn(D, generator=g, device=DEV)
        s["q_weight"] = 1 + 0.2 * torch.randn(D, generator=g, device=DEV)
        if case["packed"]:                     # the three projections of a token behind each other
            qkv = _normal((B, new, (Hq + 2 * Hkv) * D), dt, g)
            s["q"], s["k"] = qkv[..., : Hq * D], qkv[..., Hq * D: (Hq + Hkv) * D]
        else:
            s["q"], s["k"] = _normal((B, new, Hq * D), dt, g), _normal((B, new, Hkv * D), dt, g)
        names = ["q_pos", "k_norm", "k_pos"] if case["rotate"] else ["q_norm", "k_norm"]
        for x in names:
            s[x] = torch.zeros(B, Hq if x[0] == "q" else Hkv, new, D, dtype=dt, device=DEV)
        angles = torch.arange(case["ctx"] if case["rotate"] else 1, dtype=torch.float64, device=DEV)[:, None] * inv
        s["cos_pos"], s["sin_pos"] = angles.cos().float(), angles.sin().float()
        if own:
            from paper_2502_12665_amd import binding as lib
            s["dims"] = lib.make_dims(B, Hq, Hkv, D, 16, case["ctx"], stride)
        return s
    # The cache: [lead][kv][rows of it]; pages of a pool, or sequences.
    lead, rows = (B * slots + 3, page) if page else (B, stride)
    s["page_table"] = torch.randperm(lead, generator=g, device=DEV)[: B * slots].reshape(B, slots).int().contiguous() if page else None
    s["rows"] = torch.empty(lead, Hkv, rows, D, dtype=torch.uint8, device=DEV)
    s["scales"] = torch.empty(lead, Hkv, rows, 2 * D // GROUP, dtype=torch.uint8, device=DEV)
    some = max(1, (1 << 18) // (Hkv * rows))   # pages (or sequences) drawn at a time
    for i in range(0, lead, some):
        shape = (min(some, lead - i), Hkv, rows, D)
        s["rows"][i:i + some], s["scales"][i:i + some] = _cached(_normal(shape, torch.float32, g), _normal(shape, torch.float32, g))
    s["bounds"] = None
    if kind == "step" or (kind == "write" and case["bounds"]):
        # The smallest and largest of blk normal values lie about z sigma around the block's own mean.
        z = math.sqrt(2 * math.log(blk)) - 0.6
        mid = 0.4 * torch.randn((lead, Hkv, rows // blk, D), generator=g, device=DEV)
        half = z * (0.8 + 0.4 * torch.rand(mid.shape, generator=g, device=DEV))
        s["bounds"] = torch.stack([(mid - half).to(dt), (mid + half).to(dt)], 3)
    if kind in ("write", "step"):
        s["k_new"], s["v_new"] = _normal((B, Hkv, new, D), dt, g), _normal((B, Hkv, new, D), dt, g)
    if kind in ("write", "read"):
        s["k_out"], s["v_out"] = (torch.zeros(B, Hkv, new, D, dtype=dt, device=DEV) for _ in range(2))
    angles = 2048 * inv
    s["cos_b"], s["sin_b"] = angles.cos().float(), angles.sin().float()
    angles = torch.arange(max(w, 1), dtype=torch.float64, device=DEV)[:, None] * inv
    s["cos_win"], s["sin_win"] = angles.cos().float(), angles.sin().float()
    if kind in ("attend", "step"):
        heads, k = Hkv if case["shared"] else Hq, case["n_sel"]
        s["q"] = _normal((B, Hq, D), dt, g)
        s["out"] = torch.empty(B, Hq, D, dtype=dt, device=DEV)
        if kind == "attend":   # a selection as the calls before it leave it: ascending, -1 behind the last
            s["q_rot"] = _rotated(s["q"], s["cos_b"], s["sin_b"])
            lo, hi = _candidates(_tokens_of(s), case)
            size = blk if case["unit"] == "blocks" else 1
            first, last = lo // size, torch.where(hi > lo, (hi + size - 1) // size, lo // size)
            total = -(-case["ctx"] // size)
            at = torch.arange(total, device=DEV)
            keys = torch.rand((B, heads, total), generator=g, device=DEV)
            keys.masked_fill_(((at < first[:, None]) | (at >= last[:, None]))[:, None], 2.0)
            count = (last - first).clamp(max=k)[:, None].expand(B, heads)
            pick = keys.argsort(-1)[..., :k]
            pick = torch.nn.functional.pad(pick, (0, k - pick.shape[-1]), value=total)
            pick = torch.where(torch.arange(k, device=DEV) < count[..., None], pick, 1 << 30).sort(-1).values
            s["sel_idx"] = torch.where(pick < 1 << 30, pick, -1).int().contiguous()
            s["sel_count"] = count.int().contiguous()
        else:
            s["q_rot"] = torch.empty(B, Hq, D, device=DEV)
            s["sel_idx"] = torch.empty(B, heads, k, dtype=torch.int32, device=DEV)
            s["sel_count"] = torch.empty(B, heads, dtype=torch.int32, device=DEV)
    if own:   # the library's handle on the cache and its workspace, which a program makes once
        from paper_2502_12665_amd import binding as lib
        s["dims"] = lib.make_dims(B, Hq, Hkv, D, 16, case["ctx"], stride)
        s["cache"] = lib.Kv4Cache(s["dims"], blk, dt, s["rows"], s["scales"], bounds=s["bounds"], page_table=s["page_table"], page_size=page)
        attended = case["n_sel"] * (blk if case["unit"] == "blocks" else 1)
        size = max(256, lib.workspace_bytes(s["dims"], lib.OP_BLOCK_TOPK), lib.workspace_bytes(s["dims"], lib.OP_ATTN_KV4, attended, w))
        s["ws"] = torch.empty(size, dtype=torch.uint8, device=DEV)
    return s


# ---------------------------------------------------------------------------------------------- plain forms

def _tokens_of(s):
    c = s["case"]
    return s["seq_lens"].long() if s["seq_lens"] is not None else torch.full((c["batch"],), c["ctx"], dtype=torch.long, device=DEV)


def _new_of(s):
    """How many of each sequence's tokens a call is about, its last ones."""
    new = _tokens_of(s).clamp(max=s["case"]["new"])
    return new if s["new_lens"] is None else torch.minimum(new, s["new_lens"].long())


def _candidates(n, case):
    """First and one past the last position that competes: neither a sink nor in the window."""
    hi = (n.long() - case["window"]).clamp(min=0)
    return hi.clamp(max=case["sink"]), hi


def _rotated(x, cos, sin):
    """The pairs (t, t + 64) turned by the angles of cos / sin, in float64, rounded once."""
    a, b = x[..., :HALF].double(), x[..., HALF:].double()
    return torch.cat([a * cos.double() - b * sin.double(), b * cos.double() + a * sin.double()], -1).float()


def _place(s, pos, size):
    """Number of the piece of `size` tokens that holds position pos [B, Hkv, ...] in the cache's memory."""
    c = s["case"]
    b = torch.arange(c["batch"], device=DEV).reshape((-1,) + (1,) * (pos.dim() - 1))
    h = torch.arange(c["kv_heads"], device=DEV).reshape((1, -1) + (1,) * (pos.dim() - 2))
    if c["page"]:
        page = s["page_table"].long()[b, pos // c["page"]]
        return (page * c["kv_heads"] + h) * (c["page"] // size) + pos % c["page"] // size
    return (b * c["kv_heads"] + h) * (s["stride"] // size) + pos // size


def _values(s, row):
    """Keys and values that cached rows (their numbers [...]) stand for, float32."""
    table = torch.tensor(E2M1 + tuple(-x for x in E2M1), device=DEV)
    bytes_, scales = s["rows"].view(-1, D)[row], s["scales"].view(-1, 8)[row]
    scale = torch.where(scales > 0, torch.exp2(scales.float() - 127), 0.0).repeat_interleave(GROUP, -1)
    k = torch.stack([bytes_[..., :HALF] & 15, bytes_[..., :HALF] >> 4], -1).flatten(-2)
    v = bytes_[..., HALF:].unflatten(-1, (16, 4)).transpose(-1, -2).flatten(-2)
    v = torch.stack([v & 15, v >> 4], -1).flatten(-2)
    return table[k.long()] * scale[..., :D], table[v.long()] * scale[..., D:]


def _norm_plain(s):
    c = s["case"]
    new = _new_of(s)
    there = torch.arange(c["new"], device=DEV) < new[:, None]                      # [B, new]
    pos = ((_tokens_of(s) - new)[:, None] + torch.arange(c["new"], device=DEV)).clamp(0, s["cos_pos"].shape[0] - 1)
    out = {}
    for x in ("q", "k"):
        y = s[x].unflatten(-1, (-1, D)).transpose(1, 2).float()                    # [B, H, new, D]
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * s[x + "_weight"]
        keep = there[:, None, :, None]
        if x + "_norm" in s:
            out[x + "_norm"] = torch.where(keep, y, 0.0).to(s[x].dtype)
        if x + "_pos" in s:
            cos, sin = s["cos_pos"][pos][:, None], s["sin_pos"][pos][:, None]
            a, b = y[..., :HALF], y[..., HALF:]
            out[x + "_pos"] = torch.where(keep, torch.cat([a * cos - b * sin, b * cos + a * sin], -1), 0.0).to(s[x].dtype)
    return out


def _append_plain(s):
    c = s["case"]
    B, Hkv, blk, n_new = c["batch"], c["kv_heads"], c["block"], c["new"]
    n, new = _tokens_of(s), _new_of(s)
    start = n - new
    at = torch.arange(n_new, device=DEV)
    there = (at < new[:, None])[:, None].expand(B, Hkv, n_new)
    row = _place(s, (start[:, None] + at).clamp(max=s["stride"] - 1)[:, None].expand(B, Hkv, n_new), 1)
    rows, scales = _cached(s["k_new"], s["v_new"])
    s["rows"].view(-1, D)[row[there]] = rows[there]
    s["scales"].view(-1, 8)[row[there]] = scales[there]
    if s["bounds"] is None:
        return
    first = start // blk                                                           # the first block that gets tokens
    nb = (n_new + blk - 1) // blk + 1
    pos = (first * blk)[:, None] + torch.arange(nb * blk, device=DEV)              # [B, nb * blk]
    fresh = ((pos >= start[:, None]) & (pos < n[:, None])).reshape(B, 1, nb, blk, 1)
    take = (pos - start[:, None]).clamp(0, n_new - 1)
    keys = s["k_new"].gather(2, take[:, None, :, None].expand(B, Hkv, nb * blk, D)).float().reshape(B, Hkv, nb, blk, D)
    block = first[:, None] + torch.arange(nb, device=DEV)
    where = _place(s, (block * blk).clamp(max=s["stride"] - blk)[:, None].expand(B, Hkv, nb), blk)
    lo, hi = torch.where(fresh, keys, math.inf).amin(3), torch.where(fresh, keys, -math.inf).amax(3)
    bounds = s["bounds"].view(-1, 2, D)
    before = bounds[where].float()
    had = (start[:, None] > block * blk)[:, None, :, None]                         # tokens from before
    lo = torch.where(had, torch.minimum(lo, before[..., 0, :]), lo)
    hi = torch.where(had, torch.maximum(hi, before[..., 1, :]), hi)
    t = ((block * blk < n[:, None]) & (new > 0)[:, None])[:, None].expand(B, Hkv, nb)
    bounds[where[t]] = torch.stack([lo, hi], 3)[t].to(bounds.dtype)


def _read_plain(s):
    c = s["case"]
    B, Hkv, n_new = c["batch"], c["kv_heads"], c["new"]
    n, new = _tokens_of(s), _new_of(s)
    at = torch.arange(n_new, device=DEV)
    there = (at < new[:, None])[:, None, :, None]
    row = _place(s, ((n - new)[:, None] + at).clamp(max=s["stride"] - 1)[:, None].expand(B, Hkv, n_new), 1)
    k, v = _values(s, row)
    return {"k": torch.where(there, k, 0.0).to(s["k_out"].dtype), "v": torch.where(there, v, 0.0).to(s["v_out"].dtype)}


def _select_plain(s):
    c = s["case"]
    B, Hq, Hkv, blk, k = c["batch"], c["heads"], c["kv_heads"], c["block"], c["n_sel"]
    q_rot = _rotated(s["q"], s["cos_b"], s["sin_b"])
    lo, hi = _candidates(_tokens_of(s), c)
    nb = -(-c["ctx"] // blk)
    block = torch.arange(nb, device=DEV)
    first, last = lo // blk, torch.where(hi > lo, (hi + blk - 1) // blk, lo // blk)
    live = (block >= first[:, None]) & (block < last[:, None])
    bounds = s["bounds"].view(-1, 2, D)[_place(s, (block * blk).expand(B, Hkv, nb), blk)].double()   # [B, Hkv, nb, 2, D]
    q = q_rot.double().reshape(B, Hkv, Hq // Hkv, D)
    # max(q lo, q hi) is q hi for q > 0 and q lo for q < 0
    score = q.clamp(min=0) @ bounds[..., 1, :].transpose(-1, -2).contiguous()
    score += q.clamp(max=0) @ bounds[..., 0, :].transpose(-1, -2).contiguous()
    score = score.sum(2) if c["shared"] else score.reshape(B, Hq, nb)
    score = torch.where(live[:, None], score.float(), -math.inf)
    order = score.sort(dim=-1, descending=True, stable=True).indices[..., :k]
    count = (last - first).clamp(max=k)[:, None].expand(score.shape[:2])
    order = torch.nn.functional.pad(order, (0, k - order.shape[-1]))
    valid = torch.arange(k, device=DEV) < count[..., None]
    idx = torch.where(valid, order, 1 << 30).sort(-1).values
    return q_rot, torch.where(valid, idx, -1).int(), count.int()


def _attend_plain(s, q_rot, sel_idx, sel_count):
    c = s["case"]
    B, Hq, Hkv, blk, w = c["batch"], c["heads"], c["kv_heads"], c["block"], c["window"]
    n = _tokens_of(s)
    lo, hi = _candidates(n, c)
    heads = sel_idx.shape[1]
    idx = sel_idx.long()
    valid = torch.arange(idx.shape[-1], device=DEV) < sel_count[..., None]
    if c["unit"] == "blocks":
        idx = (idx[..., None] * blk + torch.arange(blk, device=DEV)).flatten(-2)
        valid = valid.repeat_interleave(blk, -1)
    valid = valid & (idx >= lo[:, None, None]) & (idx < hi[:, None, None])
    sink = torch.arange(c["sink"], device=DEV).expand(B, heads, c["sink"])
    recent = (hi[:, None, None] + torch.arange(w, device=DEV)).expand(B, heads, w)
    pos = torch.cat([sink, idx, recent], -1)
    valid = torch.cat([sink < lo[:, None, None], valid, recent < n[:, None, None]], -1)
    pos = torch.where(valid, pos, 0)
    S = pos.shape[-1]
    keys, vals = (x.reshape(B, heads, S, D) for x in _values(s, _place(s, pos.reshape(B, Hkv, -1), 1)))
    q = q_rot.reshape(B, heads, -1, D)                     # [B, heads, 1 or G, D]
    far = S - w
    logit = q @ keys[:, :, :far].transpose(-1, -2)
    if w:
        delta = (n[:, None] - 1 - hi[:, None] - torch.arange(w, device=DEV)).clamp(0, w - 1)
        turned = _rotated(s["q"][:, :, None], s["cos_win"][delta][:, None], s["sin_win"][delta][:, None])   # [B, Hq, w, D]
        near = (turned.reshape(B, heads, -1, w, D) * keys[:, :, None, far:]).sum(-1)
        logit = torch.cat([logit, near], -1)
    del keys
    logit = torch.where(valid[:, :, None], logit / math.sqrt(D), -math.inf)
    top = logit.amax(-1, keepdim=True)
    p = (logit - torch.where(top > -math.inf, top, 0.0)).exp()
    total = p.sum(-1, keepdim=True)
    out = (p @ vals) / torch.where(total > 0, total, 1.0)
    return out.reshape(B, Hq, D).to(s["q"].dtype)


def run(state):
    s, c = state, state["case"]
    kind = c["kind"]
    if not own:
        if kind == "norm":
            return _norm_plain(s)
        if kind == "attend":
            return {"out": _attend_plain(s, s["q_rot"], s["sel_idx"], s["sel_count"])}
        if kind in ("write", "step"):
            _append_plain(s)
        if kind == "step":
            q_rot, idx, count = _select_plain(s)
            return {"out": _attend_plain(s, q_rot, idx, count), "idx": idx, "count": count}
        out = _read_plain(s)
        if kind == "write" and s["bounds"] is not None:
            out["bounds"] = s["bounds"]
        return out
    from paper_2502_12665_amd import binding as lib
    if kind == "norm":
        lib.qk_norm_rope(s["dims"], s["q"], s["k"], c["new"], s["q_weight"], s["k_weight"], EPS, s["cos_pos"] if c["rotate"] else None,
                         s["sin_pos"] if c["rotate"] else None, s["seq_lens"], s["new_lens"], q_norm=s.get("q_norm"),
                         k_norm=s.get("k_norm"), q_pos=s.get("q_pos"), k_pos=s.get("k_pos"))
        return {x: s[x] for x in ("q_norm", "k_norm", "q_pos", "k_pos") if x in s}
    if kind in ("write", "step"):
        lib.kv4_append(s["dims"], s["cache"], s["k_new"], s["v_new"], c["new"], s["seq_lens"], s["new_lens"])
    if kind in ("write", "read"):
        lib.kv4_read(s["dims"], s["cache"], c["new"], s["seq_lens"], s["new_lens"], s["k_out"], s["v_out"])
        out = {"k": s["k_out"], "v": s["v_out"]}
        if kind == "write" and s["bounds"] is not None:
            out["bounds"] = s["bounds"]
        return out
    if kind == "step":
        lib.block_topk(s["dims"], s["cache"].blocks, s["q"], s["cos_b"], s["sin_b"], s["q_rot"], c["shared"], c["n_sel"], c["window"],
                       c["sink"], s["seq_lens"], s["sel_idx"], s["sel_count"], ws=s["ws"])
    lib.sparse_attn_kv4(s["dims"], s["cache"], s["q"], s["q_rot"], s["sel_idx"], s["sel_count"], c["n_sel"],
                        c["block"] if c["unit"] == "blocks" else 1, c["shared"], c["window"], c["sink"], s["cos_win"], s["sin_win"],
                        s["seq_lens"], s["out"], s["ws"])
    return {"out": s["out"]} if kind == "attend" else {"out": s["out"], "idx": s["sel_idx"], "count": s["sel_count"]}


# ---------------------------------------------------------------------------------------------- what it takes

def work(case):
    """Every sequence counted with `ctx` tokens (a ragged batch has about two thirds of that).  Rows that several heads of a KV head
    select count once, as many as independent selections have in common."""
    B, Hq, Hkv, blk, ctx, w = case["batch"], case["heads"], case["kv_heads"], case["block"], case["ctx"], case["window"]
    kind, e, row = case["kind"], 2 if case["dtype"] == "bf16" else 4, D + 8
    share = 2 / 3 if case["ragged"] else 1.0
    tokens = B * min(case["new"], ctx) * (0.6 if case["ragged"] and case["new"] > 1 else 1.0)
    moved = flops = 0.0
    if kind == "norm":
        written = Hq + 2 * Hkv if case["rotate"] else Hq + Hkv
        moved += tokens * ((Hq + Hkv + written) * D * e + (HALF * 8 if case["rotate"] else 0))
        flops += tokens * (Hq + Hkv) * D * (7 if case["rotate"] else 4)
    if kind in ("write", "step"):
        moved += tokens * Hkv * (2 * D * e + row)
        if case["bounds"]:
            moved += 2 * D * e * max(tokens * Hkv / blk, B * Hkv)
        flops += 2 * tokens * Hkv * D * 3
    if kind in ("write", "read"):
        moved += tokens * Hkv * (2 * D * e + (row if kind == "read" else 0))
        flops += 2 * tokens * Hkv * D
    candidates = max(1, share * ctx - w - case["sink"])
    heads = Hkv if case["shared"] else Hq
    if kind == "step":
        blocks = B * candidates / blk
        moved += Hkv * blocks * 2 * D * e + B * heads * case["n_sel"] * 8 + B * Hq * D * (e + 4)
        flops += Hq * blocks * 2 * D
    if kind in ("attend", "step"):
        size = blk if case["unit"] == "blocks" else 1
        far = min(case["n_sel"] * size, candidates)
        recent = min(w + case["sink"], ctx)
        rows = candidates * (1 - (1 - far / candidates) ** (heads // Hkv))
        moved += B * Hkv * (rows + recent) * row + B * heads * (far / size) * 4 + B * Hq * D * (2 * e + 4)
        flops += 4 * D * B * Hq * (far + recent)
    return {"bytes": moved, "flops": flops}


# ---------------------------------------------------------------------------------------------- in 64 bits

def _rounded64(x):
    """The values that rows x [..., 128] (float64) stand for in 4 bits."""
    grid = torch.tensor(E2M1, dtype=torch.float64, device=DEV)
    x = x.unflatten(-1, (D // GROUP, GROUP))
    a = x.abs().amax(-1, keepdim=True)
    scale = torch.exp2(torch.ceil(torch.log2(a.clamp(min=TINY) / 6) - 1e-12))
    y = x.abs() / scale
    up = torch.bucketize(y, grid).clamp(max=7)             # the first number that is not below
    down = (up - 1).clamp(min=0)
    over, under = grid[up] - y, y - grid[down]
    pick = torch.where((over < under) | ((over == under) & (up % 2 == 0)), up, down)
    return torch.where(a < TINY, 0.0, torch.sign(x) * grid[pick] * scale).flatten(-2)


def _decoded64(s, row):
    """The same of cached rows, by their bytes."""
    bytes_, scales = s["rows"].view(-1, D)[row].long(), s["scales"].view(-1, 8)[row].double()
    nibbles = torch.stack([bytes_ % 16, bytes_ // 16], -1)                         # [..., byte, half]
    magnitude = nibbles % 8
    number = torch.where(magnitude < 2, magnitude / 2.0, (1 + (magnitude % 2) / 2.0) * 2.0 ** (magnitude // 2 - 1).double())
    number = torch.where(nibbles >= 8, -number, number)
    d = torch.arange(D, device=DEV)
    k = number[..., d // 2, d % 2] * torch.pow(2.0, scales[..., d // GROUP] - 127)
    at = HALF + 4 * (d % GROUP // 2) + d // GROUP
    v = number[..., at, d % 2] * torch.pow(2.0, scales[..., 4 + d // GROUP] - 127)
    return k, v


def _row_at(s, b, h, pos):
    """Memory rows of positions pos of one sequence and KV head."""
    c = s["case"]
    if c["page"]:
        return (s["page_table"][b].long()[pos // c["page"]] * c["kv_heads"] + h) * c["page"] + pos % c["page"]
    return (b * c["kv_heads"] + h) * s["stride"] + pos


def _turn64(x, cos, sin):
    a, b = x[..., :HALF], x[..., HALF:]
    return torch.cat((a * cos - b * sin, a * sin + b * cos), dim=-1)


def _lens(s):
    c = s["case"]
    n = [c["ctx"]] * c["batch"] if s["seq_lens"] is None else s["seq_lens"].tolist()
    m = [c["new"]] * c["batch"] if s["new_lens"] is None else s["new_lens"].tolist()
    return [(b, n[b], min(m[b], c["new"], n[b])) for b in range(c["batch"])]


def _exact_norm(s):
    c = s["case"]
    out = {x: torch.zeros(s[x].shape, dtype=torch.float64, device=DEV) for x in ("q_norm", "k_norm", "q_pos", "k_pos") if x in s}
    for b, n, m in _lens(s):
        for x, heads in (("q", c["heads"]), ("k", c["kv_heads"])):
            for h in range(heads):
                y = s[x][b, :m, h * D:(h + 1) * D].double()
                y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / D + EPS) * s[x + "_weight"].double()
                if x + "_norm" in out:
                    out[x + "_norm"][b, h, :m] = y
                if x + "_pos" in out:
                    out[x + "_pos"][b, h, :m] = _turn64(y, s["cos_pos"][n - m:n].double(), s["sin_pos"][n - m:n].double())
    return out


def _exact_append(s, bounds):
    """Writes the rounded tokens over the float64 keys and values `s` is given, and the bounds."""
    c = s["case"]
    blk = c["block"]
    for b, n, m in _lens(s):
        for p in range((n - m) // blk * blk, n, blk) if m else ():
            part = s["k_new"][b, :, max(0, p - (n - m)):min(m, p + blk - (n - m))].double()
            edge = torch.stack([part.amin(1), part.amax(1)], 1)                    # [Hkv, 2, D]
            at = _row_at(s, b, torch.arange(c["kv_heads"], device=DEV), torch.tensor(p, device=DEV)) // blk
            if p < n - m:
                old = bounds.view(-1, 2, D)[at]
                edge = torch.stack([torch.minimum(edge[:, 0], old[:, 0]), torch.maximum(edge[:, 1], old[:, 1])], 1)
            bounds.view(-1, 2, D)[at] = edge


def _exact_select(s, bounds):
    c = s["case"]
    blk, G = c["block"], c["heads"] // c["kv_heads"]
    q = _turn64(s["q"].double(), s["cos_b"].double(), s["sin_b"].double()).float().double()
    heads = c["kv_heads"] if c["shared"] else c["heads"]
    idx = torch.full((c["batch"], heads, c["n_sel"]), -1, dtype=torch.long, device=DEV)
    for b, n, _ in _lens(s):
        hi = max(0, n - c["window"])
        lo = min(c["sink"], hi)
        if hi <= lo:
            continue
        blocks = torch.arange(lo // blk, (hi + blk - 1) // blk, device=DEV)
        for h in range(c["kv_heads"]):
            bd = bounds.view(-1, 2, D)[_row_at(s, b, h, blocks * blk) // blk]
            # the middle plus the half width seen by |q|
            mid, half = (bd[:, 0] + bd[:, 1]) / 2, (bd[:, 1] - bd[:, 0]) / 2
            qq = q[b, h * G:(h + 1) * G]
            sc = qq @ mid.t().contiguous() + qq.abs() @ half.t().contiguous()
            sc = sc.sum(0, keepdim=True) if c["shared"] else sc
            k = min(c["n_sel"], len(blocks))
            o = h if c["shared"] else h * G
            idx[b, o:o + sc.shape[0], :k] = blocks[sc.topk(k, -1).indices.sort(-1).values]
    return q, idx


def _exact_attend(s, q_rot, idx):
    c = s["case"]
    blk, G, w = c["block"], c["heads"] // c["kv_heads"], c["window"]
    out = torch.zeros(c["batch"], c["heads"], D, dtype=torch.float64, device=DEV)
    for b, n, m in _lens(s):
        hi = max(0, n - w)
        lo = min(c["sink"], hi)
        near = torch.arange(hi, n, device=DEV)
        for h in range(c["heads"]):
            kv = h // G
            sel = idx[b, kv if c["shared"] else h].long()
            sel = sel[sel >= 0]
            if c["unit"] == "blocks":
                sel = (sel[:, None] * blk + torch.arange(blk, device=DEV)).reshape(-1)
                sel = sel[(sel >= lo) & (sel < hi)]
            far = torch.cat([torch.arange(lo, device=DEV), sel])
            pos = torch.cat([far, near])
            if pos.numel() == 0:
                continue
            k64, v64 = _decoded64(s, _row_at(s, b, kv, pos))
            if c["kind"] == "step":                        # the step's own token
                k64 = torch.where((pos >= n - m)[:, None], _rounded64(s["k_new"][b, kv, :m].double()), k64)
                v64 = torch.where((pos >= n - m)[:, None], _rounded64(s["v_new"][b, kv, :m].double()), v64)
            delta = n - 1 - near
            turned = _turn64(s["q"][b, h].double(), s["cos_win"][delta].double(), s["sin_win"][delta].double())
            logit = torch.cat([k64[: len(far)] @ q_rot[b, h].double(), (k64[len(far):] * turned).sum(-1)]) / D ** 0.5
            out[b, h] = torch.softmax(logit, 0) @ v64
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "norm":
        return _exact_norm(s)
    if kind == "attend":
        return {"out": _exact_attend(s, s["q_rot"], s["sel_idx"])}
    bounds = None if s["bounds"] is None else s["bounds"].double()
    if kind in ("write", "step") and bounds is not None:
        _exact_append(s, bounds)
    if kind == "step":
        q, idx = _exact_select(s, bounds)
        return {"out": _exact_attend(s, q, idx), "idx": None, "count": None}
    out = {x: torch.zeros(s[x + "_out"].shape, dtype=torch.float64, device=DEV) for x in ("k", "v")}
    for b, n, m in _lens(s):
        for h in range(case["kv_heads"]):
            if kind == "write":
                k64, v64 = _rounded64(s["k_new"][b, h, :m].double()), _rounded64(s["v_new"][b, h, :m].double())
            else:
                k64, v64 = _decoded64(s, _row_at(s, b, h, torch.arange(n - m, n, device=DEV)))
            out["k"][b, h, :m], out["v"][b, h, :m] = k64, v64
    if kind == "write" and bounds is not None:
        out["bounds"] = bounds
    return out
