"""The lengths of the shared-prefix attention's ranges (the plan, compiled for the host)."""
import numpy as np
import pytest

from test_prefix_plan import CASES, _plan, rules  # noqa: F401

LONGEST = 1 << 19  # keys over which O, rounded once for 16 of them, may be off by 2^-10


@pytest.mark.parametrize("hist,new,prefix,heads,mla", CASES + [
    ([1 << 20], [2000], 0, 16, False),
    ([1 << 20], [4096], 0, 128, True),                        # tiles that would be whole
    ([(1 << 20) + 5, 700], [4096, 1], 0, 128, True),
    ([1 << 20] * 32, [1] * 32, (1 << 20) - 3, 16, True),      # the shared part
    ([(1 << 21) + 300] * 16, [1] * 16, 1 << 21, 8, False),
    ([1 << 19] * 300, [1] * 300, (1 << 19) - 100, 128, True),
    ([(1 << 30) - 8], [8], 0, 1, False),                      # more ranges than the plan weighs up
    ([(1 << 30) - 4000], [4000], 0, 128, True),
    ([(1 << 30) - 1] * 3, [1] * 3, 1 << 29, 4, False),
])
def test_no_range_is_longer(rules, hist, new, prefix, heads, mla):  # noqa: F811
    p, blocks, ctx = _plan(rules, hist, new, prefix, heads, mla)
    own = max(ctx) - p["prefix"]
    assert (p["shared_chunks"] == 0 or p["chunk"] <= LONGEST) and p["chunk"] % 32 == 0
    assert p["shared_chunks"] * p["chunk"] >= p["prefix"]
    if p["whole"]:
        assert own <= LONGEST
    if p["own_tiles"] > p["whole"]:
        assert p["chunk"] <= LONGEST and p["own_chunks"] * p["chunk"] >= own
    assert p["slots"] in (1, p["shared_chunks"] + p["own_chunks"]) and p["blocks"] == len(blocks)
    assert len(set(map(tuple, blocks.tolist()))) == len(blocks)
    assert np.all(blocks[:, 3] < p["slots"])
