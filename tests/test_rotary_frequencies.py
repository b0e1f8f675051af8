"""The stretched rotary frequencies, pair by pair (host only)."""
import math

import numpy as np
import pytest

import paper_2609_36938_amd as janus


def _want(dim, base, factor, first, last):
    """Pairs up to `first` kept, from `last` on divided by factor, a straight line in the pair's number between."""
    j = np.arange(dim // 2)
    own = base ** (-2.0 * j / dim)
    share = np.clip((j - first) / (last - first), 0, 1)
    return own * (1 - share) + own / factor * share


@pytest.mark.parametrize("dim,base,factor,ctx,fast,slow,first,last", [
    # 4096 positions are 4096 / 2 pi base^(-2 j / dim) turns: 32 of them at j = 10.47, one at 22.51
    (64, 10000.0, 40.0, 4096, 32.0, 1.0, 10, 23),
    (128, 10000.0, 8.0, 4096, 32.0, 1.0, 20, 46),       # 20.94 and 45.03
    (64, 500000.0, 4.0, 8192, 32.0, 1.0, 9, 18),        # 9.04 and 17.49
    (16, 10000.0, 2.0, 64, 32.0, 1.0, 0, 3),            # below 0, and 2.02
    (32, 100.0, 16.0, 100000, 32.0, 1.0, 21, 31),       # 21.58, and 33.61: the last element's number
])
def test_the_ramp(dim, base, factor, ctx, fast, slow, first, last):
    at = [dim * math.log(ctx / (2 * math.pi * t)) / (2 * math.log(base)) for t in (fast, slow)]
    assert max(math.floor(at[0]), 0) == first and min(math.ceil(at[1]), dim - 1) == last  # the comments' numbers
    freq, mag = janus.rotary_frequencies(dim, base, "yarn", factor, ctx, fast, slow)
    assert np.allclose(freq, _want(dim, base, factor, first, last), rtol=1e-13, atol=0)
    assert mag == np.float32(0.1 * math.log(factor) + 1)


def test_a_ramp_of_one_step():
    """Both ends just behind pair 12: it and those before are kept, the ones behind are stretched."""
    dim, base = 64, 10000.0
    ctx = 4096
    turns = ctx / (2 * math.pi) * base ** (-2 * 12.0 / dim)  # of pair 12, over the original context
    freq, _ = janus.rotary_frequencies(dim, base, "yarn", 8.0, ctx, turns * (1 - 1e-9), turns * (1 - 2e-9))
    own = base ** (-2.0 * np.arange(dim // 2) / dim)
    kept = np.isclose(freq, own, rtol=1e-13, atol=0)
    assert kept[:13].all() and not kept[13:].any() and np.allclose(freq[13:], own[13:] / 8, rtol=1e-13, atol=0)
