"""janus_prefix_attn against dense attention in 64 bits.

Tolerances.  Inputs are bf16, so products are exact in fp32; a logit's sum over the dims
is within dqk * 2^-24 of the sum of its terms' magnitudes (`size`), and its scaling adds two
roundings: d = (dqk + 2) * 2^-24 * size, by which each probability, the sum and lse may be off
(exponentials and logarithm: 2^-20 more, lse in its own size).  Probabilities go into the product in bf16 (2^-8 of
each).  An output is therefore within (2^-8 + 2 d + 2^-18) * sum p |v| of the
exact one, and its own rounding to bf16 adds 2^-8 of its value."""
import numpy as np
import pytest
import torch

from plain import attention

pytestmark = pytest.mark.gpu
janus = pytest.importorskip("paper_2609_36938_amd")


class Case:
    def __init__(self, hist, new, heads, kind, prefix, page, es=0, seed=0, copy=True, stride=0, q_std=1.0, scale=None):
        rng = np.random.default_rng(seed)
        self.hist, self.new, self.prefix, self.page, self.es = list(hist), list(new), prefix, page, es
        self.dqk, self.dv = (576, 512) if kind == "mla" else (128, 128)
        self.bt = janus.Batch(hist, new, entry_shift=es)
        ctx = [(m + n) >> es for m, n in zip(hist, new)]
        shared = prefix // page
        pages = [max(-(-c // page), shared if shared * page <= c else -(-c // page)) for c in ctx]
        order = rng.permutation(shared + sum(pages) + 9)
        self.table = np.zeros((len(ctx), max(1, -(-max(ctx) // page))), np.int32)
        at = shared
        for b, n in enumerate(pages):
            own = min(shared, n)
            self.table[b, :own] = order[:own]
            self.table[b, own:n] = order[at:at + n - own]
            at += n - own
        rows = (shared + sum(pages) + 9) * page
        width = self.dqk + stride
        t = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).bfloat16()  # noqa: E731
        self.k = t(rows, width)
        self.v = self.k if kind != "mqa2" else t(rows, self.dv + stride)
        self.q = (t(sum(new), heads, self.dqk).float() * q_std).bfloat16()
        self.scale = scale if scale is not None else 1 / np.sqrt(self.dqk)
        if prefix % page and copy:  # sessions' copies of the page that the prefix ends in
            ids = np.arange(shared * page, prefix)
            src = self.rows_of(0, ids)
            for b in range(1, len(ctx)):
                n = max(0, min(len(ids), ctx[b] - shared * page))
                for pool in {id(self.k): self.k, id(self.v): self.v}.values():
                    pool[self.rows_of(b, ids[:n])] = pool[src[:n]]

    def rows_of(self, b, ids):
        return self.table[b][ids // self.page].astype(np.int64) * self.page + ids % self.page

    def run(self, prefix=None, **kw):
        k = self.k.cuda()
        v = k if self.v is self.k else self.v.cuda()
        return janus.prefix_attn(self.bt, self.q.cuda(), k, v, torch.from_numpy(self.table).cuda(), self.page,
                                 self.prefix if prefix is None else prefix, float(self.scale), dv=self.dv,
                                 want_lse=True, **kw)

    def check(self, out, lse, keep=None, **kw):
        d = lambda t: t.double().numpy()  # noqa: E731
        want, wl, mass, size = attention(d(self.q), d(self.k)[:, :self.dqk], d(self.v)[:, :self.dv], self.hist, self.new,
                                         self.rows_of, self.scale, self.es, **kw)
        off = (self.dqk + 2) * 2.0 ** -24 * size
        tol = (2.0 ** -8 + 2 * off[..., None] + 2.0 ** -18) * mass
        if out.dtype == torch.bfloat16:
            tol = tol + 2.0 ** -8 * np.abs(want)
        err = np.abs(out.double().cpu().numpy() - want)
        sel = slice(None) if keep is None else keep
        assert (err <= tol)[sel].all(), (err - tol)[sel].max()
        got = lse.double().cpu().numpy()
        none = np.isneginf(wl)
        assert np.array_equal(np.isneginf(got)[sel], none[sel])
        ok = ~none
        ltol = np.where(ok, off + 2.0 ** -20 + 2.0 ** -22 * np.abs(np.where(ok, wl, 0)), 0)
        assert (np.abs(np.where(ok, got, 0) - np.where(ok, wl, 0)) <= ltol)[sel].all()


SHAPES = [
    # hist, new, heads, kind, prefix, page
    ([0], [1], 16, "mla", 0, 64),
    ([5, 0, 64], [3, 1, 70], 16, "mla", 0, 64),
    ([300, 301, 331], [1, 1, 1], 128, "mla", 300, 64),      # a prefix that ends inside a page and a tile
    ([256] * 9, [1] * 9, 16, "mla", 256, 64),               # nothing but the prefix and the token itself
    ([1000, 1040, 1500], [2, 1, 5], 32, "mla", 1000, 16),   # pages shorter than a tile
    ([130, 200], [7, 40], 5, "mla", 97, 1),                 # pages of one row, heads that straddle tiles
    ([500] * 40, [1] * 40, 1, "mla", 500, 128),
    ([700], [150], 128, "mla", 700, 64),
    ([0], [1], 1, "mqa2", 0, 64),
    ([0, 3], [200, 1], 8, "mqa2", 0, 64),
    ([700, 705, 900, 701], [1, 1, 3, 2], 8, "mqa2", 699, 64),
    ([2000] * 17, [1] * 17, 16, "mqa", 2000, 32),           # K and V in one pool
    ([333, 400], [100, 31], 3, "mqa2", 330, 2),
    ([900] * 3, [1, 0, 1], 128, "mqa2", 512, 64),           # a session that appends nothing
    ([40, 1000, 2000], [1, 1, 1], 8, "mqa2", 40, 64),       # sessions of very different lengths
]


@pytest.mark.parametrize("hist,new,heads,kind,prefix,page", SHAPES)
def test_shapes(hist, new, heads, kind, prefix, page):
    print("prefix", hist[:4], new[:4], heads, kind, prefix, page, flush=True)
    c = Case(hist, new, heads, kind, prefix, page, stride=0 if heads % 2 else 8)
    c.check(*c.run())
    c.check(*c.run(out_dtype="f32"))
    if prefix:                                   # the same batch, nothing declared common
        c.check(*c.run(prefix=0))


@pytest.mark.parametrize("kind", ["mla", "mqa2"])
@pytest.mark.parametrize("es,hist,new", [(3, [100, 5, 64], [3, 2, 9]), (7, [1000, 127], [40, 1])])
def test_entries(kind, es, hist, new):
    """Entries of 2^e tokens; a session's first tokens may have none."""
    c = Case(hist, new, 16, kind, 0, 4, es=es)
    c.check(*c.run())
    p = min((m + n) >> es for m, n in zip(hist, new))
    if p > 0:
        c = Case(hist, new, 16, kind, p, 4, es=es)
        c.check(*c.run())


@pytest.mark.parametrize("kind", ["mla", "mqa2"])
def test_sessions_shorter_than_the_prefix(kind):
    """Tokens that end inside the prefix attend to what they have of it."""
    c = Case([400, 90, 399, 0], [1, 12, 1, 1], 16, kind, 380, 64, copy=True)
    c.check(*c.run())


@pytest.mark.parametrize("kind", ["mla", "mqa2"])
@pytest.mark.parametrize("scale", [-0.3, 0.0, 4.0])
def test_scales(kind, scale):
    """A scale of either sign, none, and logits that move the maximum again and again."""
    c = Case([300, 280], [3, 1], 16, kind, 250, 64, scale=scale, q_std=2.0 if scale > 1 else 1.0)
    c.check(*c.run(out_dtype="f32"))


@pytest.mark.parametrize("kind", ["mla", "mqa2"])
@pytest.mark.parametrize("heads", [16, 128, 7])
def test_what_is_masked_does_not_matter(kind, heads):
    """NaN and infinities in rows that a token does not attend to: later appended tokens' rows, rows of the pool that no
    session has, ids behind the last one, and table entries that are not used."""
    c = Case([290, 330], [20, 12], heads, kind, 200, 64)
    used = np.zeros(len(c.k), bool)
    for b in range(2):
        used[c.rows_of(b, np.arange(c.hist[b] + c.new[b]))] = True
    bad = torch.tensor([float("nan"), float("inf"), float("-inf")]).bfloat16()
    for pool in {id(c.k): c.k, id(c.v): c.v}.values():
        idle = np.flatnonzero(~used)
        pool[idle] = bad[torch.from_numpy(idle % 3)][:, None]
        late = c.rows_of(0, np.arange(300, 310))  # session 0's tokens 10 .. 19
        pool[late] = bad[torch.from_numpy(np.arange(10) % 3)][:, None]
    got = c.run(out_dtype="f32")
    early = np.r_[0:10, 20:32]
    c.check(*got, keep=early)
    assert not torch.isfinite(got[0][10:20]).any()


@pytest.mark.parametrize("kind", ["mla", "mqa2"])
def test_an_infinity_goes_where_it_is_attended_to(kind):
    """Single values of V: +inf, -inf and NaN in dims of their own, in a row that the later tokens read."""
    c = Case([64], [40], 4, kind, 0, 64)
    row = int(c.rows_of(0, np.array([80]))[0])
    v = c.v
    if kind == "mla":                              # K and V are one row: a query of 0 there keeps the logits
        c.q[:, :, :3] = 0
    v[row, :3] = torch.tensor([float("inf"), float("-inf"), float("nan")]).bfloat16()
    if kind == "mla":                              # 0 * inf is NaN in the logits of the tokens that read it
        got = c.run(out_dtype="f32")[0]
        assert torch.isfinite(got[:16]).all() and torch.isnan(got[16:]).all()
        return
    got, lse = c.run(out_dtype="f32")
    v[row, :3] = 0                                 # the other dims, and the tokens before, are as without them
    mask = got.clone()
    mask[16:, :, :3] = c.run(out_dtype="f32")[0][16:, :, :3]
    c.check(mask, lse)
    assert (got[16:, :, 0] == float("inf")).all() and (got[16:, :, 1] == float("-inf")).all()
    assert torch.isnan(got[16:, :, 2]).all()


def test_rows_behind_the_last_session_stay():
    c = Case([300, 310], [3, 2], 16, "mla", 300, 64)
    q = torch.cat([c.q, c.q])
    bt = c.bt
    for kind in (300, 0):
        bt.total_q = bt.c.total_q = 5
        want = c.run(prefix=kind)
        bt.total_q = bt.c.total_q = 10
        out = torch.full((10, 16, 512), 3.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((10, 16), 3.0, device="cuda")
        k = c.k.cuda()
        janus.prefix_attn(bt, q.cuda(), k, k, torch.from_numpy(c.table).cuda(), 64, kind, float(c.scale), dv=512, out=out,
                          lse=lse)
        assert (out[5:] == 3).all() and (lse[5:] == 3).all()
        c.check(out[:5], lse[:5])
        c.check(*want)


def test_long_contexts_in_ranges():
    """Few rows over long contexts: split over many blocks."""
    c = Case([20000, 20100], [1, 1], 16, "mqa2", 20000, 64)
    c.check(*c.run())
    c = Case([9000], [1], 16, "mla", 0, 64)
    c.check(*c.run())


@pytest.mark.parametrize("kind,heads,hist,new,tokens", [
    ("mla", 128, [1500, 1300], [150, 160], [0, 100, 149, 150, 255, 256, 257, 300, 309]),
    ("mqa2", 16, [2000, 0], [3900, 601], [0, 7, 2000, 3899, 3900, 4095, 4096, 4097, 4103, 4104, 4400, 4500]),
])
def test_whole_rounds_and_a_split_rest(kind, heads, hist, new, tokens):
    """More tiles than blocks run at a time: the first ones whole, the last ones in ranges."""
    c = Case(hist, new, heads, kind, 0, 64)
    print("prefix rest", kind, flush=True)
    c.check(*c.run(), keep=np.array(tokens), tokens=set(tokens))


def test_two_captured_calls_share_no_state():
    """Two calls captured into one graph with workspaces of their own, replayed; every replay equals the eager call."""
    a, b = Case([600, 620], [1, 1], 16, "mla", 600, 64), Case([900], [3], 8, "mqa2", 0, 64, seed=2)
    args = []
    for c in (a, b):
        k = c.k.cuda()
        args.append((c.bt, c.q.cuda(), k, k if c.v is c.k else c.v.cuda(), torch.from_numpy(c.table).cuda(), c.page, c.prefix,
                     float(c.scale)))
    outs = [torch.empty((c.bt.total_q, c.q.shape[1], c.dv), dtype=torch.bfloat16, device="cuda") for c in (a, b)]
    ws = [torch.empty(64 << 20, dtype=torch.uint8, device="cuda") for _ in range(2)]
    calls = lambda: [janus.prefix_attn(*x, dv=c.dv, out=o, workspace=w) for x, c, o, w in zip(args, (a, b), outs, ws)]  # noqa: E731
    calls()
    torch.cuda.synchronize()
    want = [o.clone() for o in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(3):
        for o, w in zip(outs, ws):
            o.fill_(7)
            w.fill_(0x7f)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))


def test_workspace_too_small():
    c = Case([20000], [1], 16, "mqa2", 0, 64)
    with pytest.raises(janus.JanusError, match="workspace too small"):
        c.run(workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("kind,page", [("mla", 64), ("mla", 4), ("mqa2", 16)])
def test_far_pages(kind, page):
    """Rows beyond 2^32 bytes of a pool hold what rows at its beginning hold: the same result, bit by bit."""
    c = Case([300, 333, 1000], [1, 1, 2], 16, kind, 300, page)
    want = c.run(out_dtype="f32")
    near = c.k.cuda()
    width, rows = near.shape[-1], near.numel() // near.shape[-1]
    total = -(-(5 << 30) // (2 * width)) // page * page
    print("prefix far", kind, page, total, flush=True)
    pools = []
    for p in (c.k, c.v) if c.v is not c.k else (c.k,):
        far = torch.empty((total, width), dtype=torch.bfloat16, device="cuda")
        far[total - rows:] = p.cuda().view(rows, width)
        pools.append(far)
    table = torch.from_numpy(c.table).cuda()
    table = torch.where(table >= 0, table + (total - rows) // page, table)
    got = janus.prefix_attn(c.bt, c.q.cuda(), pools[0], pools[-1], table, page, c.prefix, float(c.scale), dv=c.dv,
                            out_dtype="f32", want_lse=True)
    for g, w in zip(got, want):
        assert torch.equal(g, w)


def test_queries_beyond_32_bits():
    """More than 2^31 elements of q: the last sessions get what they get in a batch of their own."""
    B, H, last = 30000, 128, 50
    hist = np.arange(B) % 5
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    q = torch.randn((B, H, 576), generator=g, device="cuda", dtype=torch.bfloat16)
    kv = torch.randn((64 * 16, 576), generator=g, device="cuda", dtype=torch.bfloat16)
    table = torch.randint(0, 64, (B, 1), generator=g, device="cuda", dtype=torch.int32)
    print("prefix many queries", q.numel(), flush=True)
    got = janus.prefix_attn(janus.Batch(hist, [1] * B), q, kv, kv, table, 16, 0, 0.04, dv=512)[0]
    want = janus.prefix_attn(janus.Batch(hist[-last:], [1] * last), q[-last:].contiguous(), kv, kv,
                             table[-last:].contiguous(), 16, 0, 0.04, dv=512)[0]
    assert q.numel() > 2**31 and torch.equal(got[-last:], want) and float(want.abs().max()) > 0.1


@pytest.mark.parametrize("kind,hist,new", [("mla", [300], [70]), ("mla", [5000], [1]), ("mqa2", [300], [70]), ("mqa2", [5000], [1])])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_outputs_at_four_bytes(kind, hist, new, dt):
    """An output that begins at any word: the results of an aligned one, and nothing before or behind them."""
    c = Case(hist, new, 16, kind, 0, 64)
    want, lse = c.run(out_dtype=dt)
    skip = 2 if dt == "bf16" else 1
    buf = torch.full((want.numel() + 2 * skip,), 7, dtype=want.dtype, device="cuda")
    lbuf = torch.full((lse.numel() + 2,), 7, dtype=torch.float32, device="cuda")
    out, got = c.run(out_dtype=dt, out=buf[skip:-skip].view(want.shape), lse=lbuf[1:-1].view(lse.shape))
    assert torch.equal(out, want) and torch.equal(got, lse)
    assert (buf[:skip] == 7).all() and (buf[-skip:] == 7).all() and lbuf[0] == 7 and lbuf[-1] == 7


@pytest.mark.parametrize("kind", ["mla", "mqa2"])
def test_replays_with_shorter_sessions(kind):
    """A captured call reads the lengths on the device: up to those it was made for, each replay has the lengths
    of its time."""
    c = Case([900, 1500, 700], [1, 2, 1], 16, kind, 500, 64)
    args = (c.q.cuda(), *(t.cuda() for t in (c.k, c.v)), torch.from_numpy(c.table).cuda(), 64, 500, float(c.scale))
    if c.v is c.k:
        args = (args[0], args[1], args[1], *args[3:])
    call = lambda bt: janus.prefix_attn(bt, *args, dv=c.dv, out_dtype="f32", want_lse=True)  # noqa: E731
    call(c.bt)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = call(c.bt)
    for hist in ([900, 1500, 700], [501, 640, 500], [899, 64, 0]):
        c.bt.hist_len.copy_(torch.tensor(hist, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        c.hist = hist
        c.check(out, lse)


def test_strides_of_their_own():
    """K and V as halves of one row, and pools of different strides: what two plain pools give, bit by bit."""
    c = Case([700, 705, 900], [1, 30, 2], 8, "mqa2", 699, 16)
    want = c.run(out_dtype="f32")
    n = c.k.shape[0]
    both = torch.cat([c.k, c.v], 1).cuda()
    k, v = torch.zeros((n, 136), dtype=torch.bfloat16), torch.zeros((n, 1024), dtype=torch.bfloat16)
    k[:, :128], v[:, 512:640] = c.k, c.v
    k, v = k.cuda(), v.cuda()
    table = torch.from_numpy(c.table).cuda()
    for kp, vp, ks, vs in ((both, both[:, 128:], 256, 256), (k, v[:, 512:], 136, 1024)):
        got = janus.prefix_attn(c.bt, c.q.cuda(), kp, vp, table, 16, 699, float(c.scale), k_row_stride=ks, v_row_stride=vs,
                                dv=128, out_dtype="f32", want_lse=True)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
