"""The shared-prefix attention's plan, compiled for the host: its blocks give every (row, key) to exactly one
block, and every split row's ranges to slots of their own."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_36938_amd", "csrc")
WRAP = r"""
#include "launch_rules.hpp"
using namespace janus;
extern "C" void plan(int n, int total_q, int max_q, int max_ctx, long total_ctx, int prefix, int heads, int mla, long *o)
{
    const PrefixPlan p = prefix_plan(n, total_q, max_q, max_ctx, total_ctx, prefix, heads, mla);
    const long v[] = {p.prefix, p.chunk, p.shared_tiles, p.shared_chunks, p.own_tiles, p.own_chunks, p.whole, p.alike,
                      p.slots, (long)p.part_rows, (long)p.blocks, p.one};
    for (int i = 0; i < 12; ++i)
        o[i] = v[i];
}
extern "C" void blocks(int n, int total_q, int max_q, int max_ctx, long total_ctx, int prefix, int heads, int mla, int *o)
{
    const PrefixPlan p = prefix_plan(n, total_q, max_q, max_ctx, total_ctx, prefix, heads, mla);
    for (int b = 0; b < p.blocks; ++b) {
        const PrefixBlock k = prefix_block(p, b);
        o[4 * b] = k.shared, o[4 * b + 1] = k.tile, o[4 * b + 2] = k.chunk, o[4 * b + 3] = k.slot;
    }
}
extern "C" int first(int q, int heads, int s) { return prefix_tile_first(q, heads, s); }
"""
NAMES = "prefix chunk shared_tiles shared_chunks own_tiles own_chunks whole alike slots part_rows blocks one".split()


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "r.cpp").write_text(WRAP)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-shared", "-fPIC", "-I", CSRC, str(d / "r.cpp"), "-o",
                           str(d / "r.so")])
    return ctypes.CDLL(str(d / "r.so"))


def _plan(rules, hist, new, prefix, heads, mla, es=0, max_q=None):
    ctx = [(m + n) >> es for m, n in zip(hist, new)]
    args = (len(hist), sum(new), max_q or max(new), max(ctx), ctypes.c_long(sum(ctx)), prefix, heads, int(mla))
    o = (ctypes.c_long * 12)()
    rules.plan(*args, o)
    p = dict(zip(NAMES, o))
    b = (ctypes.c_int * (4 * p["blocks"]))()
    rules.blocks(*args, b)
    return p, np.array(b, dtype=np.int64).reshape(-1, 4), ctx


CASES = [
    ([4096 + 200] * 16, [1] * 16, 4096, 8, False),
    ([131072 + 1000] * 32, [1] * 32, 131072, 16, True),
    ([32768 + 16, 36000] * 32, [1] * 64, 32768, 128, True),
    ([16384] * 8, [100, 300, 200, 150, 250, 123, 211, 280], 16384, 128, True),
    ([0], [1], 0, 1, False),
    ([131072], [1], 0, 128, True),
    ([600, 0, 900], [3, 0, 700], 0, 5, False),
    ([5000, 90, 100], [2100, 2000, 1], 64, 16, False),
    ([700] * 300, [1] * 300, 640, 16, True),
    ([2000], [300], 0, 128, True),
    ([30000, 31000], [2000, 1500], 30000, 16, False),
    ([900, 40, 2000, 900], [2, 0, 8, 1], 0, 16, True),
    ([900, 940, 2000, 900], [8, 0, 8, 0], 900, 16, False),
    ([5000] * 3, [1, 2, 1], 0, 64, True),
]


@pytest.mark.parametrize("hist,new,prefix,heads,mla", CASES)
@pytest.mark.parametrize("more", [0, 1000])  # a bound on the tokens of a session that is not tight
def test_every_row_and_key_once(rules, hist, new, prefix, heads, mla, more):
    p, blocks, ctx = _plan(rules, hist, new, prefix, heads, mla, max_q=max(new) + more)
    assert p["one"] == (heads % 128 != 0 and (max(new) + more) * heads <= 128)
    q = np.concatenate([[0], np.cumsum(new)])
    rows = int(q[-1]) * heads
    first = [s if p["one"] else rules.first(int(q[s]), heads, s) for s in range(len(hist) + 1)]
    assert first.pop() == p["own_tiles"]
    assert len(set(map(tuple, blocks))) == len(blocks) and p["chunk"] % 32 == 0
    seen = np.zeros(rows, np.int64)      # keys that blocks give the row
    slots = {}
    last = np.repeat([m for m in hist], new) + np.concatenate([np.arange(n) for n in new]) + 1
    last = np.repeat(last, heads)        # keys that the row has
    for shared, tile, chunk, slot in blocks:
        if shared:
            r0, r1 = tile * 128, min(tile * 128 + 128, rows)
            k0, k1 = chunk * p["chunk"], min((chunk + 1) * p["chunk"], p["prefix"])
            part = r0
        else:
            s = max(i for i in range(len(hist)) if first[i] <= tile)
            r0 = int(q[s]) * heads + (tile - first[s]) * 128
            r1 = min(r0 + 128, int(q[s + 1]) * heads)
            k0 = p["prefix"] + chunk * p["chunk"]
            k1 = 1 << 30 if slot < 0 else k0 + p["chunk"]
            part = r0 if p["prefix"] else (tile - p["whole"]) * 128
        if r0 >= r1:
            continue
        assert (slot < 0) == (not shared and tile < p["whole"]) and slot < p["slots"]
        if slot >= 0:
            for r in range(r0, r1):
                assert slots.setdefault((slot, part + r - r0), r) == r and part + r - r0 < p["part_rows"]
        have = np.clip(np.minimum(last[r0:r1], k1) - k0, 0, None)
        seen[r0:r1] += have
    assert np.array_equal(seen, last)
    if p["slots"] > 1:                   # a split row has all slots
        split = {at for _, at in slots}
        assert len(slots) == len(split) * p["slots"]
    # blocks of one XCD are neighbours, none is lost
    assert p["blocks"] == len(blocks)


def test_what_the_plan_aims_at(rules):
    # heads of all sessions together where they do not fill a block apart, and only there
    assert _plan(rules, [9000] * 32, [1] * 32, 8192, 16, True)[0]["prefix"] == 8192
    assert _plan(rules, [9000] * 32, [1] * 32, 8192, 128, True)[0]["prefix"] == 0
    assert _plan(rules, [9000], [1], 8192, 16, True)[0]["prefix"] == 0
    # whole rounds are not split
    p = _plan(rules, [16384] * 8, [213] * 8, 16384, 128, True)[0]
    assert p["whole"] == 8 * 213 // 256 * 256 and p["slots"] > 1
    assert _plan(rules, [16384] * 8, [32] * 8, 16384, 128, True)[0]["slots"] == 1
    # no CU without a block because of tiles that may be empty
    assert _plan(rules, [131072 + 1000] * 32, [1] * 32, 131072, 16, True)[0]["blocks"] == 256
    # one long row: many blocks
    assert _plan(rules, [131072], [1], 0, 128, True)[0]["blocks"] > 100
