"""The operators together, as a layer's step uses them: pages for the appended tokens, their rows into the bf16 and
fp8 caches and the indexer's keys, queries rotated, then the selection path and the dense attention over what was written.

With k at least the context the selection is everything, so sparse_attn and prefix_attn give the same attention: each
is held to the 64-bit form of the cache's own contents (read back), prefix_attn by its derived tolerance and the path's
calls by theirs (2e-2, absolute and of the row's largest output).  The cache's contents themselves are held to the
formula by the operators' own tests."""
import threading

import numpy as np
import pytest
import torch

from plain import attention, page_grow

pytestmark = pytest.mark.gpu
janus = pytest.importorskip("paper_2609_36938_amd")

PAGE, HEADS, PREFIX = 64, 16, 200


class Layer:
    """Sessions on one prompt, their caches and one step's projections."""

    def __init__(self, hist, new, seed=0):
        rng = np.random.default_rng(seed)
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.t = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()
        self.hist, self.new, T = hist, new, sum(new)
        self.bt = janus.Batch(hist, new)
        B, shared = len(hist), PREFIX // PAGE
        had = [-(-h // PAGE) for h in hist]
        width = max(-(-(h + n) // PAGE) for h, n in zip(hist, new))
        self.pages = 300
        order = rng.permutation(self.pages).astype(np.int32)
        self.table0 = np.full((B, width), -1, np.int32)
        at = shared
        for b in range(B):
            self.table0[b, :shared] = order[:shared]
            self.table0[b, shared:had[b]] = order[at:at + had[b] - shared]
            at += had[b] - shared
        self.free0 = order[at:]
        self.table, self.free = torch.from_numpy(self.table0).cuda(), torch.from_numpy(self.free0).cuda()
        self.kv = self.t(self.pages * PAGE, 576)
        for b in range(1, B):  # the sessions' copies of the page the prompt ends in
            n = PREFIX % PAGE
            self.kv[self.table0[b, shared] * PAGE:][:n] = self.kv[self.table0[0, shared] * PAGE:][:n]
        self.kv8 = torch.zeros((self.pages * PAGE, 592), dtype=torch.uint8, device="cuda")
        self.keys = self.t(self.bt.total_ctx, 128).to(torch.float8_e4m3fn).view(torch.uint8)
        self.kscale = torch.rand(self.bt.total_ctx, generator=g, device="cuda") + 0.5
        self.latent, self.joint = self.t(T, 512), self.t(T, 576)
        self.qb, self.q = self.t(T, HEADS, 192), self.t(T, HEADS, 576)
        self.qi, self.ki = self.t(T, 64, 128), self.t(T, 128)
        self.w = torch.rand((T, 64), generator=g, device="cuda") / 8
        self.rot = janus.Rotary(64, 512, "interleaved", scaling="yarn", factor=40.0, original_ctx=4096)
        self.rot_q = janus.Rotary(64, 0, "interleaved", inv_freq=self.rot.inv_freq, mscale=self.rot.mscale)
        self.rot_i = janus.Rotary(64, 0, "half")
        # the whole cache in fp8, as an earlier step would have left it
        full = janus.Batch([0], [self.pages * PAGE])
        janus.kv_append(full, self.kv, self.kv8, rows=torch.arange(self.pages * PAGE, device="cuda"))
        self.slots = torch.empty(T, dtype=torch.int64, device="cuda")
        self.counts = torch.empty(3, dtype=torch.int32, device="cuda")
        self.k = 512
        self.scale = 1 / 24.0
        self.ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")

    def step(self):
        bt = self.bt
        janus.page_grow(bt, PAGE, self.free, self.table, out=(self.slots, self.counts))
        pe = self.joint[:, 512:]
        janus.kv_append(bt, self.latent, self.kv, self.rot, pe, self.slots)
        janus.kv_append(bt, self.latent, self.kv8, self.rot, pe, self.slots)
        janus.kv_append(bt, self.ki, self.keys, self.rot_i, out_scale=self.kscale)
        janus.rope(bt, self.rot_q, self.qb[..., 128:], out=self.q[..., 512:])
        qi, qs = janus.rope(bt, self.rot_i, self.qi, out_dtype="fp8")
        scores = janus.index_scores(bt, qi, self.keys, self.w, q_scale=qs, k_scale=self.kscale)
        sel = janus.topk(bt, scores, self.k)
        sparse = janus.sparse_attn(bt, self.q, self.kv, self.kv, self.table, PAGE, sel, self.scale, dv=512,
                                   out_dtype="f32")[0]
        fp8 = janus.sparse_attn_fp8kv(bt, self.q, self.kv8, self.table, PAGE, sel, self.scale, out_dtype="f32",
                                      workspace=self.ws)[0]
        dense, lse = janus.prefix_attn(bt, self.q, self.kv, self.kv, self.table, PAGE, PREFIX, self.scale, dv=512,
                                       out_dtype="f32", want_lse=True, workspace=self.ws)
        return dict(sel=sel, sparse=sparse, fp8=fp8, dense=dense, lse=lse)


@pytest.mark.parametrize("hist,new", [([200, 255, 256, 391], [1, 1, 1, 1]), ([200, 300, 210], [70, 1, 33])])
def test_step(hist, new):
    s = Layer(hist, new)
    got = s.step()
    torch.cuda.synchronize()
    table, slots, counts = page_grow(hist, new, PAGE, 0, s.free0, 0, s.table0)
    assert np.array_equal(s.table.cpu().numpy(), table) and np.array_equal(s.slots.cpu().numpy(), slots)
    assert s.counts.tolist() == counts.tolist() and counts[2] == 0
    # k >= context: the selection is every id up to the token's own
    sel = got["sel"].cpu().numpy()
    at = 0
    for M, N in zip(hist, new):
        for i in range(N):
            assert np.array_equal(sel[at, :M + i + 1], np.arange(M + i + 1)) and (sel[at, M + i + 1:] == -1).all()
            at += 1
    rows = lambda b, ids: table[b][ids // PAGE].astype(np.int64) * PAGE + ids % PAGE  # noqa: E731
    d = lambda t: t.double().cpu().numpy()  # noqa: E731
    kv = d(s.kv)
    want, lse, mass, size = attention(d(s.q), kv, kv[:, :512], hist, new, rows, s.scale)
    off = 578 * 2.0 ** -24 * size
    assert (np.abs(d(got["dense"]) - want) <= (2.0 ** -8 + 2 * off[..., None] + 2.0 ** -18) * mass).all()
    assert (np.abs(d(got["lse"]) - lse) <= off + 2.0 ** -20 + 2.0 ** -22 * np.abs(lse)).all()
    held = d(s.kv8[:, :576].contiguous().view(torch.float8_e4m3fn)) * d(s.kv8[:, 576:580].contiguous().view(torch.float32))
    want8 = attention(d(s.q), held, held[:, :512], hist, new, rows, s.scale)[0]
    for name, ref in (("sparse", want), ("fp8", want8)):
        err = np.abs(d(got[name]) - ref).max(-1)
        assert (err <= 2e-2).all() and (err <= 2e-2 * np.abs(ref).max(-1)).all(), name


def test_step_replayed():
    """The whole step as one graph: every replay, from the caches it began with, gives the eager step's results."""
    s = Layer([200, 255, 320], [3, 1, 2], seed=4)
    first = {n: getattr(s, n).clone() for n in ("table", "kv", "kv8", "keys", "kscale", "q")}
    want = {n: t.clone() for n, t in s.step().items()}
    after = {n: getattr(s, n).clone() for n in first}
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = s.step()
    for _ in range(3):
        for n, t in first.items():
            getattr(s, n).copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(got[n], want[n]) for n in want)
        assert all(torch.equal(getattr(s, n), after[n]) for n in first)


def test_what_a_call_on_another_stream_makes_belongs_to_that_stream(monkeypatch):
    """Outputs and workspaces that a call makes itself: the allocator may give their memory to the next
    work of the stream they were made on, which has to be the launch's."""
    s, side, empty, streams = Layer([200, 255, 256, 391], [1, 1, 1, 1]), torch.cuda.Stream(), torch.empty, []
    want = s.step()["dense"].clone()
    table = s.table.clone()
    torch.cuda.synchronize()

    def seen(*args, **kw):
        streams.append(torch.cuda.current_stream().cuda_stream)
        return empty(*args, **kw)

    monkeypatch.setattr(torch, "empty", seen)
    janus.page_grow(s.bt, PAGE, s.free, table, stream=side)
    janus.rope(s.bt, s.rot_i, s.qi, out_dtype="fp8", stream=side)
    got = janus.prefix_attn(s.bt, s.q, s.kv, s.kv, s.table, PAGE, PREFIX, s.scale, dv=512, out_dtype="f32", want_lse=True,
                            stream=side)[0]
    monkeypatch.undo()
    side.synchronize()
    assert len(streams) == 2 + 2 + 3 and set(streams) == {side.cuda_stream}
    assert torch.equal(got, want)


def test_two_threads_on_streams_of_their_own():
    """Two sessions' steps at once: no call keeps anything that another one's could meet."""
    layers = [Layer([200, 255, 256, 391], [1, 1, 1, 1]), Layer([200, 300, 210], [70, 1, 33], seed=1)]
    first = [{n: getattr(s, n).clone() for n in ("table", "kv", "kv8", "keys", "kscale", "q")} for s in layers]
    want = [{n: t.clone() for n, t in s.step().items()} for s in layers]
    torch.cuda.synchronize()
    streams, got, wrong = [torch.cuda.Stream() for _ in layers], [None, None], []

    def work(i):
        try:
            with torch.cuda.stream(streams[i]):
                for _ in range(20):
                    for n, t in first[i].items():
                        getattr(layers[i], n).copy_(t)
                    got[i] = layers[i].step()
                streams[i].synchronize()
        except Exception as e:  # (of the thread: told by the test)
            wrong.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong
    for i in range(2):
        assert all(torch.equal(got[i][n], want[i][n]) for n in want[i])
