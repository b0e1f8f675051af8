"""Timed cases of the operators around the sparse-selection path: page tables
and slot maps, rotary positions, cache append, and attention for a batch with
a shared prefix.

Each case is one pass through one operator.  With `own` false it is computed in
plain torch operations; with `own` true by the library's entry points.
"""
from __future__ import annotations

import math
import zlib

import numpy as np
import torch

own = False

FP8_MAX = 448.0
FP8_ROW = 592      # bytes of an fp8 KV row: 576 values, the fp32 scale, padding
MLA, MLA_V = 576, 512
ROT = 64           # rotated dims of an MLA row and of an indexer vector


# ---- cases -----------------------------------------------------------------

def listed():
    return [
        # a decode step of 64 sessions: latency of one small call
        dict(name="pages_decode", op="pages", B=64, hist_lo=32768, hist_hi=163840, new_lo=1, new_hi=1, page=64, es=0),
        # appended prompts of a ragged batch: tens of thousands of slots
        dict(name="pages_append", op="pages", B=16, hist_lo=8192, hist_hi=65536, new_lo=512, new_hi=4096, page=64,
             es=0),
        # rotary part of the decode queries, from the projection's output into the absorbed queries
        dict(name="rope_decode_mla", op="rope", B=16, hist_lo=8192, hist_hi=49152, new_lo=1, new_hi=1, heads=128,
             kind="mla", dt="bf16", layout="interleaved", inverse=False, scaled=True),
        # the same for a long append
        dict(name="rope_append_mla", op="rope", B=1, hist_lo=131072, hist_hi=131072, new_lo=8192, new_hi=8192,
             heads=128, kind="mla", dt="bf16", layout="interleaved", inverse=False, scaled=True),
        # indexer queries: rotated, then quantised with one scale per token
        dict(name="rope_index_fp8", op="rope", B=1, hist_lo=32768, hist_hi=32768, new_lo=2048, new_hi=2048, heads=64,
             kind="index", dt="bf16", layout="half", inverse=False, scaled=False),
        # the gradient of full-width rotary heads in fp32, an odd number of tokens
        dict(name="rope_grad_f32", op="rope", B=3, hist_lo=100, hist_hi=4096, new_lo=300, new_hi=1021, heads=8,
             kind="full", dt="f32", layout="half", inverse=True, scaled=False),
        # decode: 64 new rows quantised into the fp8 cache
        dict(name="append_decode_fp8", op="append", B=64, hist_lo=32768, hist_hi=163840, new_lo=1, new_hi=1,
             kind="mla_fp8", pages=512, page=64, layout="interleaved"),
        # a long append into the bf16 cache
        dict(name="append_prefill_bf16", op="append", B=1, hist_lo=131072, hist_hi=131072, new_lo=8192, new_hi=8192,
             kind="mla_bf16", pages=256, page=64, layout="interleaved"),
        # a small batch of 8 heads with a short shared prompt
        dict(name="prefix_mqa_decode", op="prefix", B=16, heads=8, kind="mqa", prefix=4096, tail_lo=1, tail_hi=512,
             new_lo=1, new_hi=1, page=64),
        # 16 latent heads a session (a slice of the heads): the prefix is shared by all rows of a tile
        dict(name="prefix_mla16_decode", op="prefix", B=32, heads=16, kind="mla", prefix=131072, tail_lo=64,
             tail_hi=2048, new_lo=1, new_hi=1, page=64),
        # all 128 latent heads, 64 agents on one long prompt
        dict(name="prefix_mla_decode", op="prefix", B=64, heads=128, kind="mla", prefix=32768, tail_lo=16,
             tail_hi=4096, new_lo=1, new_hi=1, page=64),
        # ragged appends behind a shared prompt: the largest
        dict(name="prefix_mla_append", op="prefix", B=8, heads=128, kind="mla", prefix=16384, tail_lo=0, tail_hi=700,
             new_lo=100, new_hi=300, page=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["pages", "rope", "rope", "append", "append", "prefix", "prefix", "prefix"])
    if op == "pages":
        new = _log(rng, 1, 4096)
        return dict(op=op, B=_log(rng, 1, 600 if new < 64 else 16), hist_lo=_log(rng, 1, 4096),
                    hist_hi=_log(rng, 8192, 163840), new_lo=max(1, new // 3), new_hi=new,
                    page=rng.choice([16, 64, 128]), es=rng.choice([0, 0, 0, 3, 7]))
    if op == "rope":
        kind = rng.choice(["mla", "index", "full"])
        new = _log(rng, 1, 2048)
        return dict(op=op, B=rng.randint(1, 4) if new > 4 else _log(rng, 1, 128), hist_lo=_log(rng, 1, 4096),
                    hist_hi=_log(rng, 8192, 1000000), new_lo=max(1, new // 2), new_hi=new,
                    heads=64 if kind == "index" else rng.choice([1, 5, 8, 16, 64, 128]), kind=kind,
                    dt=rng.choice(["bf16", "f32"]), layout=rng.choice(["half", "interleaved"]),
                    inverse=kind != "index" and rng.random() < 0.3, scaled=rng.random() < 0.5)
    if op == "append":
        new = _log(rng, 1, 4096)
        return dict(op=op, B=rng.randint(1, 4) if new > 4 else _log(rng, 1, 128), hist_lo=_log(rng, 1, 4096),
                    hist_hi=_log(rng, 8192, 163840), new_lo=max(1, new // 2), new_hi=new,
                    kind=rng.choice(["mla_fp8", "mla_bf16", "index_fp8"]), pages=rng.randint(300, 600), page=64,
                    layout=rng.choice(["half", "interleaved"]))
    kind = rng.choice(["mqa", "mla"])
    new = rng.choice([1, 1, _log(rng, 2, 100)])
    heads = rng.choice([1, 4, 8, 16]) if kind == "mqa" else rng.choice([16, 32, 64, 128])
    return dict(op=op, B=_log(rng, 1, 64 if new == 1 else 8), heads=heads, kind=kind,
                prefix=_log(rng, 64, 65536 if new == 1 else 8192), tail_lo=rng.randint(0, 30),
                tail_hi=_log(rng, 40, 2000), new_lo=max(1, new // 2), new_hi=new, page=rng.choice([16, 64]))


# ---- inputs ------------------------------------------------------------------

def _lengths(c):
    """History and appended lengths: drawn from the case's ranges, the same for every seed."""
    rng = np.random.default_rng(zlib.crc32(repr(sorted((k, v) for k, v in c.items() if k != "name")).encode()))
    if c["op"] == "prefix":
        hist = c["prefix"] + rng.integers(c["tail_lo"], c["tail_hi"] + 1, c["B"])
    else:
        hist = np.exp(rng.uniform(math.log(c["hist_lo"]), math.log(c["hist_hi"]), c["B"])).round()
    return hist.astype(np.int64), rng.integers(c["new_lo"], c["new_hi"] + 1, c["B"]).astype(np.int64)


def _gen(seed, k):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed << 8) + k)
    return g


def _randn(shape, seed, k, dtype=torch.bfloat16, std=1.0):
    return (torch.randn(shape, generator=_gen(seed, k), device="cuda") * std).to(dtype)


def _frequencies(dim, scaled):
    """(inv_freq in 64 bits, magnitude): base 10000, or stretched by 40 for contexts beyond
    4096 positions: fast frequencies kept, slow ones divided, a ramp between."""
    j = torch.arange(0, dim, 2, dtype=torch.float64)
    inv = 10000.0 ** (-j / dim)
    if not scaled:
        return inv.cuda(), 1.0
    at = lambda turns: dim * math.log(4096 / (2 * math.pi * turns)) / (2 * math.log(10000.0))  # noqa: E731
    low, high = max(math.floor(at(32)), 0), min(math.ceil(at(1)), dim - 1)
    ramp = ((j / 2 - low) / max(high - low, 1e-3)).clamp(0, 1)
    return (inv * (1 - ramp) + inv / 40 * ramp).cuda(), 0.1 * math.log(40.0) + 1.0


def _rotary_shape(c):
    """(heads, head size, rotated dims, first rotated dim) of a rope or append case."""
    if c["op"] == "append":
        return (1, 128, ROT, 0) if c["kind"] == "index_fp8" else (1, MLA, ROT, MLA_V)
    if c["kind"] == "index":
        return c["heads"], 128, ROT, 0
    return (c["heads"], ROT, ROT, 0) if c["kind"] == "mla" else (c["heads"], 128, 128, 0)


def prepare(case, seed):
    c = case
    hist, new = _lengths(c)
    total = int(new.sum())
    s = dict(c=c, total=total, hist=torch.from_numpy(hist).cuda(), new=torch.from_numpy(new).cuda())
    s["q_start"] = torch.cumsum(s["new"], 0) - s["new"]
    if own:
        import paper_2609_36938_amd as janus
        s["batch"] = janus.Batch(hist, new, entry_shift=c.get("es", 0))
    rng = np.random.default_rng([seed, 2])
    if c["op"] == "pages":
        ctx = (hist + new) >> c["es"]
        width = max(1, -(-int(ctx.max()) // c["page"]))
        pool = int((-(-ctx // c["page"])).sum()) + 64
        order = rng.permutation(pool).astype(np.int32)
        had = -(-(hist >> c["es"]) // c["page"])
        table = np.zeros((len(hist), width), np.int32)
        mine = np.arange(width)[None] < had[:, None]
        table[mine] = order[: int(had.sum())]
        s["table"] = torch.from_numpy(table).cuda()
        s["free"] = torch.from_numpy(order[int(had.sum()):].copy()).cuda()
        s["head"] = torch.full((1,), int(rng.integers(0, 8)), dtype=torch.int32, device="cuda")
        return s
    if c["op"] in ("rope", "append"):
        heads, size, dim, off = _rotary_shape(c)
        s["inv_freq"], s["mag"] = _frequencies(dim, c.get("scaled", False))
        if own:
            s["rotary"] = janus.Rotary(dim, offset=off, layout=c["layout"], inv_freq=s["inv_freq"], mscale=s["mag"],
                                       inverse=c.get("inverse", False))
    if c["op"] == "rope":
        dt = torch.float32 if c["dt"] == "f32" else torch.bfloat16
        if c["kind"] == "mla":
            # the projection gives 128 unrotated and 64 rotated dims a head; the rotated ones go behind the
            # 512 absorbed ones of the queries
            s["x"] = _randn((total, heads, 192), seed, 3, dt)[..., 128:]
            s["out"] = torch.zeros((total, heads, MLA), dtype=dt, device="cuda")[..., MLA_V:]
        else:
            s["x"] = _randn((total, heads, size), seed, 3, dt)
        return s
    if c["op"] == "append":
        s["x"] = _randn((total, size), seed, 3) if c["kind"] == "index_fp8" else _randn((total, MLA_V), seed, 3)
        # the rotated part is the tail of the joint projection's row
        s["x_rot"] = None if c["kind"] == "index_fp8" else _randn((total, MLA), seed, 4)[:, MLA_V:]
        if c["kind"] == "index_fp8":
            n_rows = int((hist + new).sum())
            s["rows"] = torch.from_numpy(np.concatenate(
                [o + h + np.arange(n) for o, h, n in zip(np.cumsum(hist + new) - hist - new, hist, new)])).cuda()
            s["pool"] = _randn((n_rows, size), seed, 5).to(torch.float8_e4m3fn).view(torch.uint8)
            s["scale"] = torch.rand((n_rows,), generator=_gen(seed, 6), device="cuda") + 0.5
        else:
            n_rows = c["pages"] * c["page"]
            s["rows"] = torch.from_numpy(rng.permutation(n_rows)[:total].astype(np.int64)).cuda()
            if c["kind"] == "mla_bf16":
                s["pool"] = _randn((n_rows, MLA), seed, 5)
            else:
                s["pool"] = torch.zeros((n_rows, FP8_ROW), dtype=torch.uint8, device="cuda")
                s["pool"][:, :MLA] = _randn((n_rows, MLA), seed, 5).to(torch.float8_e4m3fn).view(torch.uint8)
                s["pool"][:, MLA:MLA + 4] = (torch.rand((n_rows, 1), generator=_gen(seed, 6), device="cuda")
                                             + 0.5).view(torch.uint8)
        return s
    # prefix: the sessions' tables begin with the same pages, their own pages follow
    page, ctx = c["page"], hist + new
    shared = c["prefix"] // page
    pages = -(-ctx // page)
    pool = shared + int((pages - shared).sum())
    order = rng.permutation(pool).astype(np.int32)
    table = np.zeros((len(ctx), int(pages.max())), np.int32)
    table[:, :shared] = order[:shared]
    table[:, shared:][np.arange(table.shape[1] - shared)[None] < (pages - shared)[:, None]] = order[shared:]
    dqk, dv = (MLA, MLA_V) if c["kind"] == "mla" else (128, 128)
    s["k"] = _randn((pool * page, dqk), seed, 3)
    s["v"] = s["k"] if c["kind"] == "mla" else _randn((pool * page, dv), seed, 4)
    s["q"] = _randn((total, c["heads"], dqk), seed, 5)
    if c["prefix"] % page:  # the page the prefix ends in: each session has its own copy of the shared rows
        first = torch.from_numpy(table[:, shared].astype(np.int64)).cuda() * page
        rows = torch.arange(c["prefix"] % page, device="cuda")
        for pool_ in ([s["k"]] if c["kind"] == "mla" else [s["k"], s["v"]]):
            pool_[first[:, None] + rows] = pool_[first[0] + rows].clone()
    s["table"] = torch.from_numpy(table).cuda()
    s["max_new"], s["max_tail"] = int(new.max()), int(ctx.max()) - c["prefix"]
    s["softmax_scale"], s["dv"] = 1.0 / math.sqrt(dqk), dv
    return s


# ---- plain forms ---------------------------------------------------------------

def _tokens(s):
    """(session, index in its append, position) of every appended token."""
    sess = torch.repeat_interleave(torch.arange(len(s["new"]), device="cuda"), s["new"], output_size=s["total"])
    i = torch.arange(s["total"], device="cuda") - s["q_start"][sess]
    return sess, i, s["hist"][sess] + i


def _pages_plain(s):
    c, table, free = s["c"], s["table"], s["free"]
    page, es = c["page"], c["es"]
    had = ((s["hist"] >> es) + page - 1) // page
    need = (((s["hist"] + s["new"]) >> es) + page - 1) // page
    fresh = need - had
    first = s["head"] + torch.cumsum(fresh, 0) - fresh
    j = torch.arange(table.shape[1], device="cuda")
    at = first[:, None] + j - had[:, None]
    mine = (j >= had[:, None]) & (j < need[:, None])
    table = torch.where(mine, free[at.clamp(0, len(free) - 1)], table)
    sess, i, pos = _tokens(s)
    entry = ((pos + 1) >> es) - 1
    done = ((pos + 1) & ((1 << es) - 1)) == 0
    e = entry.clamp(min=0)
    slots = torch.where(done, table[sess, e // page].long() * page + e % page, -1)
    taken = fresh.sum()
    counts = torch.stack([taken, s["head"][0] + taken, torch.zeros_like(taken)]).int()
    return table, slots, counts


def _rotate(s, x, pos):
    """x [tokens, heads, dim] in 32 bits, rotated; angles in 64."""
    angle = pos.double()[:, None] * s["inv_freq"]
    sign = -1.0 if s["c"].get("inverse", False) else 1.0
    cos = (angle.cos() * s["mag"]).float()[:, None]
    sin = (angle.sin() * (s["mag"] * sign)).float()[:, None]
    if s["c"]["layout"] == "half":
        a, b = x.chunk(2, -1)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)


def _quantise(x):
    """Rows of x in fp8 with a scale each."""
    flat = x.flatten(1)
    scale = flat.abs().amax(1).clamp(min=1e-12) / FP8_MAX
    return (flat / scale[:, None]).to(torch.float8_e4m3fn).view(x.shape), scale


def _rope_plain(s):
    c, x = s["c"], s["x"].float()
    _, _, dim, _ = _rotary_shape(c)
    y = torch.cat([_rotate(s, x[..., :dim], _tokens(s)[2]), x[..., dim:]], -1)
    if c["kind"] == "index":
        return _quantise(y)
    if c["kind"] == "mla":
        s["out"].copy_(y)
        return s["out"]
    return y.to(s["x"].dtype)


def _append_plain(s):
    c, pos = s["c"], _tokens(s)[2]
    if c["kind"] == "index_fp8":
        x = s["x"].float()
        row = torch.cat([_rotate(s, x[:, None, :ROT], pos)[:, 0], x[:, ROT:]], -1)
        q, scale = _quantise(row)
        s["pool"][s["rows"]] = q.view(torch.uint8)
        s["scale"][s["rows"]] = scale
        return
    row = torch.cat([s["x"].float(), _rotate(s, s["x_rot"].float()[:, None], pos)[:, 0]], -1)
    if c["kind"] == "mla_bf16":
        s["pool"][s["rows"]] = row.bfloat16()
        return
    q, scale = _quantise(row)
    s["pool"][s["rows"], :MLA] = q.view(torch.uint8)
    s["pool"][s["rows"], MLA:MLA + 4] = scale[:, None].view(torch.uint8)


def _pool_out(s):
    """The cache as what it holds: bf16 rows, or fp8 values and their scales."""
    if s["c"]["kind"] == "mla_bf16":
        return s["pool"]
    if s["c"]["kind"] == "index_fp8":
        return s["pool"].view(torch.float8_e4m3fn), s["scale"]
    return s["pool"].view(torch.float8_e4m3fn)[:, :MLA], s["pool"][:, MLA:MLA + 4].view(torch.float32)


def _rows_of(table, ids, page):
    """Pool rows of ids [..., n] through table rows [..., pages]."""
    return torch.gather(table, -1, ids // page).long() * page + ids % page


def _prefix_plain(s):
    c, table = s["c"], s["table"].long()
    page, prefix, H, dv = c["page"], c["prefix"], c["heads"], s["dv"]
    B, T, N, S = len(s["hist"]), s["total"], s["max_new"], s["max_tail"]
    q = s["q"].float() * s["softmax_scale"]
    sess, i, pos = _tokens(s)
    shared = _rows_of(table[0], torch.arange(prefix, device="cuda"), page)
    # the shared keys, for all rows at once
    near = q.view(T * H, -1) @ s["k"][shared].float().T
    # each session's own keys: padded to the longest
    ids = (prefix + torch.arange(S, device="cuda")).expand(B, S)
    inside = ids < (s["hist"] + s["new"])[:, None]
    rows = _rows_of(table, torch.where(inside, ids, 0), page)
    k = s["k"][rows].float()
    padded = torch.zeros((B, N, H, q.shape[-1]), device="cuda")
    padded[sess, i] = q
    far = torch.bmm(padded.view(B, N * H, -1), k.transpose(1, 2).contiguous()).view(B, N, H, S)[sess, i]
    far = far.masked_fill((ids[0] > pos[:, None])[:, None], -math.inf).view(T * H, S)
    top = torch.maximum(near.amax(1), far.amax(1))
    near = (near - top[:, None]).exp_()
    far = (far - top[:, None]).exp_()
    total = near.sum(1) + far.sum(1)
    out = near @ s["v"][shared][:, :dv].float()
    padded = torch.zeros((B, N, H, S), device="cuda")
    padded[sess, i] = far.view(T, H, S)
    v = s["v"][rows][..., :dv].float()
    out = out + torch.bmm(padded.view(B, N * H, S), v).view(B, N, H, dv)[sess, i].reshape(T * H, dv)
    out = out / total[:, None]
    return out.view(T, H, dv).bfloat16(), (top + total.log()).view(T, H)


def run(state):
    s, op = state, state["c"]["op"]
    if own:
        import paper_2609_36938_amd as janus
        c = s["c"]
        if op == "pages":
            return janus.page_grow(s["batch"], c["page"], s["free"], s["table"], free_head=s["head"])
        if op == "rope":
            y, scale = janus.rope(s["batch"], s["rotary"], s["x"], out=s.get("out"),
                                  out_dtype="fp8" if c["kind"] == "index" else None)
            return (y.view(torch.float8_e4m3fn), scale) if c["kind"] == "index" else y
        if op == "append":
            rows = None if c["kind"] == "index_fp8" else s["rows"]
            janus.kv_append(s["batch"], s["x"], s["pool"], rotary=s["rotary"], x_rot=s["x_rot"], rows=rows,
                            out_scale=s.get("scale"))
            return _pool_out(s)
        return janus.prefix_attn(s["batch"], s["q"], s["k"], s["v"], s["table"], c["page"], c["prefix"],
                                 s["softmax_scale"], dv=s["dv"], want_lse=True)
    if op == "pages":
        return _pages_plain(s)
    if op == "rope":
        return _rope_plain(s)
    if op == "append":
        _append_plain(s)
        return _pool_out(s)
    return _prefix_plain(s)


# ---- from the definitions, in 64 bits --------------------------------------------

def exact(case, seed):
    c = case
    if c["op"] == "pages":
        return None
    s = prepare(case, seed)
    hist, new = _lengths(c)
    pos = torch.cat([torch.arange(h, h + n, dtype=torch.float64) for h, n in zip(hist, new)]).cuda()
    if c["op"] == "prefix":
        out, lse, at = [], [], 0
        table, page = s["table"].cpu().numpy(), c["page"]
        for b, (h, n) in enumerate(zip(hist, new)):
            ids = np.arange(h + n)
            rows = torch.from_numpy(table[b][ids // page].astype(np.int64) * page + ids % page).cuda()
            k, v = s["k"][rows].double(), s["v"][rows][:, :s["dv"]].double()
            step = max(1, (1 << 28) // (len(ids) * c["heads"]))
            for i0 in range(0, int(n), step):
                m = min(step, int(n) - i0)
                logit = (s["q"][at + i0:at + i0 + m].double().reshape(m * c["heads"], -1) @ k.T) * s["softmax_scale"]
                logit = logit.view(m, c["heads"], -1)
                limit = h + i0 + torch.arange(m, device="cuda")
                logit[(torch.arange(len(ids), device="cuda") > limit[:, None])[:, None].expand_as(logit)] = -math.inf
                z = torch.logsumexp(logit, -1)
                out.append(((logit - z[..., None]).exp().view(m * c["heads"], -1) @ v).view(m, c["heads"], -1))
                lse.append(z)
            at += int(n)
        return torch.cat(out), torch.cat(lse)
    heads, size, dim, off = _rotary_shape(c)
    if c["op"] == "rope":
        x = s["x"].double()
    else:
        x = (s["x"] if s["x_rot"] is None else torch.cat([s["x"], s["x_rot"]], -1)).double()[:, None]
    # the rotation as products of complex numbers
    part = x[..., off:off + dim]
    pair = part.unflatten(-1, (2, dim // 2)).transpose(-1, -2) if c["layout"] == "half" else part.unflatten(-1, (-1, 2))
    angle = pos[:, None, None] * s["inv_freq"] * (-1 if c.get("inverse", False) else 1)
    turned = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * torch.polar(torch.full_like(angle, s["mag"]),
                                                                                      angle))
    turned = (turned.transpose(-1, -2) if c["layout"] == "half" else turned).flatten(-2)
    y = torch.cat([x[..., :off], turned, x[..., off + dim:]], -1)
    amax = y.flatten(1).abs().amax(1).clamp(min=1e-12)
    if c["op"] == "rope":
        return (y * (FP8_MAX / amax)[:, None, None], amax / FP8_MAX) if c["kind"] == "index" else y
    y = y[:, 0]
    if c["kind"] == "mla_bf16":
        pool = s["pool"].double()
        pool[s["rows"]] = y
        return pool
    held, scales = _pool_out(s)
    held, scales = held.double(), scales.double()
    held[s["rows"]] = y * (FP8_MAX / amax)[:, None]
    scales[s["rows"]] = (amax / FP8_MAX).view(-1, *scales.shape[1:])
    return held, scales


# ---- the work of a pass --------------------------------------------------------

def work(case):
    c = case
    hist, new = _lengths(c)
    total = int(new.sum())
    if c["op"] == "pages":
        fresh = int((-(-((hist + new) >> c["es"]) // c["page"]) + (-(hist >> c["es"]) // c["page"])).sum())
        return {"bytes": 8 * c["B"] + 8 * fresh + 8 * total, "flops": 0}
    if c["op"] == "rope":
        heads, size, dim, _ = _rotary_shape(c)
        n = total * heads * size
        width = 4 if c["dt"] == "f32" else 2
        out = n + 4 * total if c["kind"] == "index" else n * width
        return {"bytes": n * width + out, "flops": total * heads * dim * 3}
    if c["op"] == "append":
        _, size, dim, _ = _rotary_shape(c)
        out = 2 * size if c["kind"] == "mla_bf16" else size + 4
        return {"bytes": total * (2 * size + out + (0 if c["kind"] == "index_fp8" else 8)), "flops": total * dim * 3}
    dqk, dv = (MLA, MLA_V) if c["kind"] == "mla" else (128, 128)
    row = 2 * (dqk if c["kind"] == "mla" else dqk + dv)
    tail = int((hist + new - c["prefix"]).sum())
    pairs = int((new * hist + new * (new + 1) // 2).sum()) * c["heads"]
    return {"bytes": row * (c["prefix"] + tail) + total * c["heads"] * (2 * dqk + 2 * dv + 4),
            "flops": 2 * (dqk + dv) * pairs}
