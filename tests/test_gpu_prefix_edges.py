"""janus_prefix_attn at its edges."""
import numpy as np
import pytest
import torch

from test_prefix_plan import _plan, rules  # noqa: F401

pytestmark = pytest.mark.gpu
janus = pytest.importorskip("paper_2609_36938_amd")


@pytest.mark.parametrize("kind,heads,hist,new", [("mqa2", 16, 524288 - 8192, 8192), ("mla", 128, 524288 - 512, 512)])
def test_the_sum_over_many_keys(rules, kind, heads, hist, new):  # noqa: F811
    """Keys that all score alike, below the first: a range of 500000 of them in one block.  Logits are exact (one
    product of powers of two), so the sum is off by its own roundings alone.  The pool is two pages."""
    dqk, dv = (576, 512) if kind == "mla" else (128, 128)
    p = _plan(rules, [hist], [new], 0, heads, kind == "mla")[0]
    assert p["whole"] == p["own_tiles"] and p["slots"] == 1
    scale, low = 2.0 ** -4, 11.0                       # logits 16 and 11, in 2^-4 * 16 * 16 and 2^-4 * 16 * 11
    k = torch.zeros((128, dqk), dtype=torch.bfloat16)
    k[:, 0] = low
    k[0, 0] = 16
    k[:, 1] = 0.75                                     # (a value, q has 0 there)
    v = k if kind == "mla" else torch.full((128, dv), 0.75, dtype=torch.bfloat16)
    q = torch.zeros((new, heads, dqk), dtype=torch.bfloat16)
    q[..., 0] = 16
    table = torch.ones((1, (hist + new) // 64), dtype=torch.int32)
    table[0, 0] = 0
    kd, vd = k.cuda(), None
    vd = kd if kind == "mla" else v.cuda()
    out, lse = janus.prefix_attn(janus.Batch([hist], [new]), q.cuda(), kd, vd, table.cuda(), 64, 0, scale, dv=dv,
                                 out_dtype="f32", want_lse=True)
    n = np.arange(hist + 1, hist + new + 1, dtype=np.float64)
    want = 16 + np.log1p((n - 1) * np.exp(low - 16))
    err = np.abs(lse.double().cpu().numpy() - want[:, None])
    # scaling a logit rounds twice (2^-23 of 16), exponentials and logarithm 2^-20, the sum's own 2^-22, lse's rounding 2^-22 of it
    assert (err <= 2.0 ** -23 * 16 * 2 + 2.0 ** -20 + 2.0 ** -22 + 2.0 ** -22 * want[:, None]).all(), err.max()
    # the value 0.75: probabilities in bf16, and O's accumulators rounded once for 16 keys
    got = out[..., 1].double().cpu().numpy()
    assert (np.abs(got - 0.75) <= (2.0 ** -8 + n[:, None] / 16 * 2.0 ** -25 + 2.0 ** -18) * 0.75).all()


@pytest.mark.parametrize("kind,heads,new", [("mqa2", 16, 8192), ("mla", 128, 512)])
def test_the_output_over_many_keys(kind, heads, new):
    """Three million keys that score alike, at half the weight of the first: bf16 holds their probabilities, so
    the output is off by the roundings of O alone, one for 16 keys of a range of at most 2^19, and by those of the
    join (2^-18 with the exponentials')."""
    dqk, dv = (576, 512) if kind == "mla" else (128, 128)
    n, scale = 3 << 20, float(np.log(2) / 80)              # logits 16 * 16 and 16 * 11: ln 2 apart
    g = torch.Generator()
    g.manual_seed(0)
    vals = (torch.rand(dv, generator=g) + 0.5).bfloat16()
    k = torch.zeros((128, dqk), dtype=torch.bfloat16)
    k[:, 0] = 11
    k[0, 0] = 16
    if kind == "mla":
        k[:, 1:dv] = vals[1:]                              # (q has 0 there)
    pools = [k.cuda()] * 2 if kind == "mla" else [k.cuda(), vals.repeat(128, 1).cuda()]
    q = torch.zeros((new, heads, dqk), dtype=torch.bfloat16)
    q[..., 0] = 16
    table = torch.ones((1, n // 64), dtype=torch.int32)
    table[0, 0] = 0
    print("prefix long", kind, flush=True)
    out, lse = janus.prefix_attn(janus.Batch([n - new], [new]), q.cuda(), *pools, table.cuda(), 64, 0, scale, dv=dv,
                                 out_dtype="f32", want_lse=True)
    want = vals.double().numpy()[1:]
    err = np.abs(out[..., 1:].double().cpu().numpy() - want) / want
    assert (err <= 2.0 ** -10 + 2.0 ** -18).all(), err.max()
    ids = np.arange(n - new, n, dtype=np.float64)
    wl = 256 * scale + np.log1p(ids / 2)
    # a logit rounds twice in its scaling (2^-23 of 3.6 with log2 e: 5.2)
    assert (np.abs(lse.double().cpu().numpy() - wl[:, None]) <= 2.0 ** -23 * 5.2 + 2.0 ** -20 + 2.0 ** -22 * (1 + wl[:, None])).all()
