"""Numbers past 32 bits are refused by the binding (no GPU): passed on, their low bits alone would arrive."""
import pytest
import torch

BIG = 1 << 32


@pytest.fixture(scope="module")
def g():
    if torch.cuda.is_available():
        pytest.skip("host checks run where no GPU can be touched")
    from paper_2606_23419_amd import grinqh
    return grinqh


@pytest.mark.parametrize("kw", [dict(heads=BIG + 8), dict(head_dim=BIG + 128), dict(page=BIG + 64), dict(n_pages=BIG + 10), dict(n_pages=10 - BIG),
                                dict(format=BIG)])
def test_a_cache(g, kw):
    with pytest.raises(ValueError, match="32 bits"):
        g.make_kv_desc(**(dict(format=g.GRINQH_KV_I4, heads=8, head_dim=128, page=64, n_pages=10) | kw))


@pytest.mark.parametrize("kw", [dict(window=BIG), dict(sinks=BIG + 4), dict(max_rows=BIG + 1), dict(max_len=BIG + 1), dict(heads=BIG + 8), dict(B=BIG + 2),
                                dict(rows=BIG + 2), dict(window=64 - BIG)])
def test_attention(g, kw):
    """A window of 2^32 tokens was none, sinks of 2^32 + 4 were 4."""
    d, a = g.make_kv_desc(g.GRINQH_KV_I4, 8, 128, 64, 10), dict(heads=8, B=2, rows=2, max_rows=1, max_len=100)
    assert g.grinqh_attend_workspace_bytes(d, **a) >= 0
    with pytest.raises(ValueError, match="32 bits"):
        g.grinqh_attend_workspace_bytes(d, **(a | kw))


def test_a_plan(g):
    for B in (BIG + 2, -BIG):
        with pytest.raises(ValueError, match="32 bits"):
            g.grinqh_kv_plan_workspace_bytes(B)
    d = g.make_kv_desc(g.GRINQH_KV_I4, 8, 128, 64, 10)
    i32, pool = torch.zeros(3, dtype=torch.int32), g.kv_pool(d, device="cpu")
    for rows in (BIG + 4, 4 - BIG):
        with pytest.raises(ValueError, match="32 bits"):
            g.grinqh_kv_plan(d, pool, g.KvBatch(i32[:2].view(2, 1), i32[:2], i32), i32[:2], rows)
    wide = i32[:1].view(1, 1).expand(1, BIG + 1)
    for batch, p in ((g.KvBatch(wide, i32[:1], i32[:2]), pool), (g.KvBatch(i32[:1].view(1, 1), i32[:1], i32[:2]), g.KvPool(wide.view(-1), pool.n_free))):
        with pytest.raises(ValueError, match="32 bits"):
            g.grinqh_kv_plan(d, p, batch, i32[:1], 4)


@pytest.mark.parametrize("shape", [(BIG, 1), (BIG + 3, 8), (1, BIG + 8)])
def test_a_norm(g, shape):
    """2^32 rows were none, and what was returned had not been written."""
    t = torch.zeros((1, 1), dtype=torch.float16).expand(shape)
    for y, h in ((t, None), (None, t), (t, t)):
        with pytest.raises(ValueError, match="32 bits"):
            g.grinqh_norm(y, h)
    for kw in (dict(pre=BIG + 1), dict(post=BIG + 1)):
        with pytest.raises(ValueError, match="32 bits"):
            g.grinqh_norm(t[:1, :1], **kw)
