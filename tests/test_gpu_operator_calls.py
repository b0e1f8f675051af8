"""How the attention calls and the operators around the path take their tensors."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
janus = pytest.importorskip("paper_2609_36938_amd")


def _randn(shape, seed, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _prefix(hist, kind, heads=16, new=None):
    """Arguments of prefix_attn for sessions with pages of their own, and its dv."""
    new = new or [1] * len(hist)
    dqk, dv = (576, 512) if kind == "mla" else (128, 128)
    pages = -(-(max(hist) + max(new)) // 64)
    order = np.random.default_rng(1).permutation(len(hist) * pages).astype(np.int32).reshape(len(hist), pages)
    k = _randn((order.size * 64, dqk), 2)
    v = k if kind == "mla" else _randn((order.size * 64, dv), 3)
    bt = janus.Batch(hist, new)
    return [bt, _randn((bt.total_q, heads, dqk), 4), k, v, torch.from_numpy(order).cuda(), 64, 0, dqk ** -0.5], dv


def _empty():
    return torch.empty(0, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("kind", ["mla", "mqa"])
def test_an_empty_workspace_of_prefix_attn(kind):
    """Enough for a batch whose keys are not split, too small for another; never a call that does nothing."""
    args, dv = _prefix([20], kind)
    want = janus.prefix_attn(*args, dv=dv, want_lse=True)
    out, lse = torch.full_like(want[0], 7), torch.full_like(want[1], 7)
    janus.prefix_attn(*args, dv=dv, out=out, lse=lse, workspace=_empty())
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    args, dv = _prefix([9000], kind)
    with pytest.raises(janus.JanusError, match="workspace too small"):
        janus.prefix_attn(*args, dv=dv, workspace=_empty())


@pytest.mark.parametrize("k,splits", [(64, 1), (2000, 8)])
def test_an_empty_workspace_of_the_split_attention(k, splits):
    """The same of sparse_attn_split and sparse_attn_fp8kv."""
    (bt, q, pool, _, table, page, _, scale), _ = _prefix([3000], "mla")
    idx = torch.arange(k, dtype=torch.int32, device="cuda")[None]
    fp8 = torch.zeros((len(pool), 592), dtype=torch.uint8, device="cuda")
    janus.kv_append(janus.Batch([0], [len(pool)]), pool, fp8, rows=torch.arange(len(pool), device="cuda"))
    calls = (lambda **kw: janus.sparse_attn_split(bt, q, pool, pool, table, page, idx, scale, splits, dv=512, **kw),
             lambda **kw: janus.sparse_attn_fp8kv(bt, q, fp8, table, page, idx, scale, splits, **kw))
    for call in calls:
        want = call()[0]
        out = torch.full_like(want, 7)
        if splits == 1:
            call(out=out, workspace=_empty())
            assert torch.equal(out, want)
        else:
            with pytest.raises(janus.JanusError, match="workspace too small"):
                call(out=out, workspace=_empty())


def test_a_workspace_with_gaps():
    """Every second byte of a buffer is no workspace, however many there are."""
    args, dv = _prefix([9000], "mqa")
    with pytest.raises(janus.JanusError, match="workspace"):
        janus.prefix_attn(*args, dv=dv, workspace=torch.empty(64 << 20, dtype=torch.uint8, device="cuda")[::2])
