"""janus_prefix_attn at its edges."""
import numpy as np
import pytest
import torch

from plain import attention
from test_gpu_prefix_attn import Case
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


# ---- values that are not finite, where rows end ----------------------------------

INF, NAN = float("inf"), float("nan")


def _like(c, got, tokens):
    """The outputs of these tokens: infinite and NaN where the 64-bit form's are, else within the tolerances of
    test_gpu_prefix_attn.py."""
    out, lse = (t.double().cpu().numpy() for t in got)
    d = lambda t: t.double().numpy()  # noqa: E731
    with np.errstate(invalid="ignore"):
        want, wl, _, size = attention(d(c.q), d(c.k)[:, :c.dqk], d(c.v)[:, :c.dv], c.hist, c.new, c.rows_of, c.scale,
                                      tokens=set(tokens))
        mass = attention(d(c.q), d(c.k)[:, :c.dqk], np.nan_to_num(d(c.v)[:, :c.dv], nan=0, posinf=0, neginf=0), c.hist,
                         c.new, c.rows_of, c.scale, tokens=set(tokens))[2]
    tokens = list(tokens)
    out, want, mass, lse, wl, size = (x[tokens] for x in (out, want, mass, lse, wl, size))
    assert np.array_equal(np.isnan(out), np.isnan(want)) and np.array_equal(np.isnan(lse), np.isnan(wl))
    inf = np.isinf(want)
    assert np.array_equal(np.isinf(out), inf) and np.array_equal(out[inf], want[inf])
    ok = np.isfinite(want)
    off = (c.dqk + 2) * 2.0 ** -24 * size
    tol = (2.0 ** -8 + 2 * off[..., None] + 2.0 ** -18) * mass + (2.0 ** -8 * np.abs(want) if got[0].dtype == torch.bfloat16 else 0)
    assert (np.abs(out[ok] - want[ok]) <= tol[ok]).all()
    return ok


def _spoil(c):
    """Values of V in two rows that the later tokens read: of one kind, of two, of both signs."""
    first, second = (int(c.rows_of(0, np.array([c.hist[0] + i]))[0]) for i in (5, 20))
    c.v[first, :5] = torch.tensor([INF, -INF, NAN, INF, 1.0]).bfloat16()
    c.v[second, :5] = torch.tensor([INF, INF, 1.0, 1.0, -INF]).bfloat16()
    c.v[second, c.dv - 1] = -INF


@pytest.mark.parametrize("out_dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind,heads,hist,new,whole", [
    ("mqa2", 8, [64], [40], False),
    ("mqa2", 3, [30], [64], False),
    ("mqa2", 8, [5], [26], True),
    ("mla", 8, [5], [26], True),
    ("mqa2", 16, [9000, 50], [40, 3], False),
    ("mqa2", 16, [70], [9000], True),
    ("mla", 16, [64], [40], False),
    ("mla", 128, [9000], [40], False),
    ("mla", 16, [70], [2100], True),
])
def test_not_finite_values(rules, kind, heads, hist, new, whole, out_dtype):  # noqa: F811
    """In whole tiles and in ranges.  The rows before the values are as without them, those behind them have them in
    their dims alone (K's own, where V is in its rows: NaN everywhere)."""
    c = Case(hist, new, heads, kind, 0, 64)
    p = _plan(rules, c.hist, c.new, 0, heads, kind == "mla")[0]
    assert (p["whole"] > 0) == whole
    _spoil(c)
    print("prefix not finite", kind, heads, hist, flush=True)
    tokens = sorted({0, 4, 5, 6, 19, 20, 21, min(39, new[0] - 1), new[0] - 1, sum(new) - 1})
    ok = _like(c, c.run(out_dtype=out_dtype), tokens)
    assert ok[:2].all() and not ok[2:-1].all()


@pytest.mark.parametrize("kind", ["mla", "mqa2"])
@pytest.mark.parametrize("scale", [-0.3, 0.0])
def test_not_finite_values_of_all_rows_at_such_scales(kind, scale):
    """What every row attends to is no matter of where rows end."""
    c = Case([300, 280], [3, 1], 16, kind, 0, 64, scale=scale)
    c.v[int(c.rows_of(0, np.array([10]))[0]), :3] = torch.tensor([INF, -INF, NAN]).bfloat16()
    _like(c, c.run(out_dtype="f32"), range(4))


@pytest.mark.parametrize("kind,heads,new", [("mla", 128, 300), ("mla", 16, 40), ("mqa2", 16, 3000), ("mqa2", 8, 40)])
def test_an_overflowed_row_of_a_long_context(kind, heads, new):
    """Such rows among 90000 ids are looked for in the last tiles, and the rows around them are not done again."""
    c = Case([90000], [new], heads, kind, 0, 64)
    _spoil(c)
    print("prefix long not finite", kind, heads, new, flush=True)
    _like(c, c.run(out_dtype="f32"), [0, 4, 5, 20, 25, new - 1])


def _shared(rules, c):  # noqa: F811
    p = _plan(rules, c.hist, c.new, c.prefix, c.q.shape[1], c.dqk == 576)[0]
    assert p["shared_tiles"] > 0 and p["prefix"] == c.prefix
    return p


def _spoil_rows(c, ids, pools):
    row = torch.from_numpy(c.rows_of(0, ids))
    bad = torch.tensor([NAN, INF, -INF]).bfloat16()[torch.arange(len(ids)) % 3]
    for pool in pools:
        pool[row] = bad[:, None]


@pytest.mark.parametrize("kind,which", [("mla", "both"), ("mqa2", "both"), ("mqa2", "v")])
@pytest.mark.parametrize("heads", [16, 5])
def test_not_finite_rows_of_a_shared_prefix(rules, kind, which, heads):  # noqa: F811
    """Prefix rows that the long sessions attend to and the short ones do not."""
    c = Case([400, 90, 399, 0], [1, 12, 1, 1], heads, kind, 380, 64)
    _shared(rules, c)
    _spoil_rows(c, np.arange(200, 209), [c.v] if which == "v" else [c.k, c.v])
    got = c.run(out_dtype="f32")
    short = np.r_[1:13, 14]
    c.check(*got, keep=short)
    assert not torch.isfinite(got[0][[0, 13]]).any()
    got = c.run()
    c.check(*got, keep=short)


@pytest.mark.parametrize("kind", ["mla", "mqa2"])
def test_many_sessions_of_a_shared_prefix(rules, kind):  # noqa: F811
    """More sessions than a block looks through at once for one shorter than the prefix."""
    hist = [700] * 300
    hist[7::60] = [100] * 5
    c = Case(hist, [1] * 300, 16, kind, 640, 64)
    _shared(rules, c)
    c.check(*c.run())
    _spoil_rows(c, np.arange(300, 306), [c.v])
    got = c.run(out_dtype="f32")
    short = np.arange(7, 300, 60)
    c.check(*got, keep=short)
    assert not np.isfinite(np.delete(got[0].cpu().numpy(), short, 0)).any()
