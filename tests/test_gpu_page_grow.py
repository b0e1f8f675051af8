"""janus_page_grow against a plain loop, exactly: page and entry edges, empty
sessions, a list that ends early, more sessions than a block scans at a time, and
replays of a captured call."""
import numpy as np
import pytest
import torch

from plain import page_grow

pytestmark = pytest.mark.gpu
janus = pytest.importorskip("paper_2609_36938_amd")


def _case(hist, new, page, es=0, spare=5, head=3, seed=0, width=0):
    rng = np.random.default_rng(seed)
    hist, new = np.asarray(hist, np.int64), np.asarray(new, np.int64)
    had = -(-(hist >> es) // page)
    need = -(-((hist + new) >> es) // page)
    pool = int(need.sum()) + 64
    order = rng.permutation(pool).astype(np.int32)
    table = np.full((len(hist), max(1, int(need.max())) + width), -7, np.int32)
    at = 0
    for b, n in enumerate(had):
        table[b, :n] = order[at:at + n]
        at += n
    free = order[at:at + max(0, head + int((need - had).sum()) + spare)]
    return hist, new, free, table


def _run(hist, new, page, es, free, head, table):
    bt = janus.Batch(hist, new, entry_shift=es)
    pt = torch.from_numpy(table).cuda()
    fh = torch.tensor([head], dtype=torch.int32, device="cuda")
    return bt, pt, fh, janus.page_grow(bt, page, torch.from_numpy(free).cuda(), pt, free_head=fh)


@pytest.mark.parametrize("hist,new,page,es", [
    ([0], [1], 64, 0),
    ([63, 64, 65], [1, 1, 1], 64, 0),
    ([0, 5, 0, 128], [64, 0, 200, 0], 64, 0),
    ([7, 100], [1, 33], 1, 0),
    ([1000, 3], [700, 2], 16, 0),
    ([0, 0, 0], [0, 0, 5], 64, 0),
    ([127, 128, 1000], [1, 127, 300], 2, 7),     # entries of 128 tokens
    ([5, 6], [1, 1], 64, 3),                     # one token completes none, none history
    ([15], [1], 64, 4),                          # the first entry
])
def test_edges(hist, new, page, es):
    hist, new, free, table = _case(hist, new, page, es)
    want = page_grow(hist, new, page, es, free, 3, table)
    got = _run(hist, new, page, es, free, 3, table)[3]
    for g, w in zip(got, want):
        assert np.array_equal(g.cpu().numpy(), w)


@pytest.mark.parametrize("n", [1, 255, 256, 257, 700, 2000])
def test_many_sessions(n):
    rng = np.random.default_rng(n)
    new = rng.integers(0, 3, n) if n % 2 else rng.integers(0, 40, n)
    new[rng.integers(n)] = 900
    hist, new, free, table = _case(rng.integers(0, 3000, n), new, 16, seed=n, width=2)
    want = page_grow(hist, new, 16, 0, free, 3, table)
    got = _run(hist, new, 16, 0, free, 3, table)[3]
    for g, w in zip(got, want):
        assert np.array_equal(g.cpu().numpy(), w)


@pytest.mark.parametrize("spare", [-1, -7, -1000])
def test_list_too_short(spare):
    hist, new, free, table = _case([10, 70, 0, 500], [200, 1, 130, 300], 64, spare=spare, width=1)
    want = page_grow(hist, new, 64, 0, free, 3, table)
    got = _run(hist, new, 64, 0, free, 3, table)[3]
    assert want[2][2] > 0
    for g, w in zip(got, want):
        assert np.array_equal(g.cpu().numpy(), w)


@pytest.mark.parametrize("hist,new", [(0, 2**31 - 1), (2**31 - 300, 299)])
def test_lengths_near_32_bits(hist, new):
    """The last block's rows, and pages rounded up, end at 2^31."""
    page, pages = 1 << 20, 1 << 11
    had = -(-hist // page)
    bt = janus.Batch([hist], [new])
    table = torch.full((1, pages), -7, dtype=torch.int32, device="cuda")
    table[0, :had] = torch.arange(had, dtype=torch.int32, device="cuda")
    free = torch.arange(had, pages, dtype=torch.int32, device="cuda")
    print("page_grow", hist, new, flush=True)
    table, slots, counts = janus.page_grow(bt, page, free, table)
    assert torch.equal(table[0], torch.arange(pages, dtype=torch.int32, device="cuda"))
    assert counts.tolist() == [pages - had, pages - had, 0]
    for a in range(0, new, 1 << 27):
        part = slots[a:a + (1 << 27)]
        assert torch.equal(part, torch.arange(hist + a, hist + a + part.numel(), device="cuda"))


def test_no_tokens():
    hist, new, free, table = _case([10, 70], [0, 0], 64)
    got = _run(hist, new, 64, 0, free, 3, table)[3]
    assert np.array_equal(got[0].cpu().numpy(), table) and got[1].numel() == 0
    assert got[2].tolist() == [0, 3, 0]


def test_rows_behind_the_last_session():
    """A batch padded to more rows than its sessions have: those get slot -1."""
    hist, new, free, table = _case([10, 70], [5, 9], 64)
    want = page_grow(hist, new, 64, 0, free, 0, table)
    bt = janus.Batch(hist, new)
    bt.total_q = bt.c.total_q = 300
    got = janus.page_grow(bt, 64, torch.from_numpy(free).cuda(), torch.from_numpy(table).cuda())
    assert np.array_equal(got[0].cpu().numpy(), want[0]) and got[2].tolist() == want[2].tolist()
    assert np.array_equal(got[1].cpu().numpy(), np.concatenate([want[1], np.full(286, -1)]))


def test_head_goes_from_call_to_call_and_replays():
    """Two calls in a row, the second from the head that the first left, captured and replayed."""
    hist, new, free, table = _case([10, 70, 333], [60, 3, 64], 16, head=0, spare=40)
    first = page_grow(hist, new, 16, 0, free, 0, table)
    hist2, new2 = hist + new, np.array([17, 30, 1])
    want = page_grow(hist2, new2, 16, 0, free, int(first[2][1]), np.pad(first[0], ((0, 0), (0, 4)), constant_values=-7))
    b1, b2 = janus.Batch(hist, new), janus.Batch(hist2, new2)
    start = torch.from_numpy(np.pad(table, ((0, 0), (0, 4)), constant_values=-7)).cuda()
    pt, fl = start.clone(), torch.from_numpy(free).cuda()
    outs = [(torch.empty(b.total_q, dtype=torch.int64, device="cuda"), torch.empty(3, dtype=torch.int32, device="cuda"))
            for b in (b1, b2)]

    def calls():
        janus.page_grow(b1, 16, fl, pt, out=outs[0])
        janus.page_grow(b2, 16, fl, pt, free_head=outs[0][1][1:2], out=outs[1])

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(3):
        pt.copy_(start)
        for s, c in outs:
            s.fill_(-9)
            c.fill_(-9)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(pt.cpu().numpy(), want[0])
        assert np.array_equal(outs[1][0].cpu().numpy(), want[1]) and outs[1][1].tolist() == want[2].tolist()
