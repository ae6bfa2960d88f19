"""Host-side checks of the cache and attention entry points (no GPU): every device call here is given arguments that
fail validation, so no kernel is launched."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def g():
    from paper_2606_23419_amd import grinqh
    return grinqh


@pytest.fixture(autouse=True)
def _no_launch():
    """A call that passes validation by mistake would launch on these pointers."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("host checks run where no GPU can be touched")


P = 0x1000


def desc(g, **kw):
    a = dict(format=g.GRINQH_KV_I8, heads=8, head_dim=128, page=64, n_pages=10) | kw
    return g.make_kv_desc(**a)


def test_struct_layouts(g):
    assert [ctypes.sizeof(t) for t in (g.KvDesc, g.AttendDesc, g._KvCache, g._KvBatch, g._Rows)] == [20, 28, 32, 40, 24]


def test_kv_bytes(g):
    assert g.grinqh_kv_bytes(desc(g)) == (10 * 8 * 64 * 128, 10 * 8 * 64 * 4)
    assert g.grinqh_kv_bytes(desc(g, format=g.GRINQH_KV_BF16, head_dim=64)) == (10 * 8 * 64 * 128, 0)
    big = desc(g, n_pages=1 << 20, page=1 << 12)
    assert g.grinqh_kv_bytes(big)[0] == 1 << 42


@pytest.mark.parametrize("kw,status", [
    (dict(format=3), -1), (dict(format=-1), -1), (dict(heads=0), -1), (dict(heads=1025), -1), (dict(head_dim=96), -2),
    (dict(head_dim=256), -2), (dict(page=0), -1), (dict(page=48), -1), (dict(page=1 << 21), -1), (dict(n_pages=0), -1),
    (dict(n_pages=1 << 30, page=1 << 20, heads=1024), -3),
])
def test_kv_desc_refusals(g, kw, status):
    with pytest.raises(g.GrinqhError) as e:
        g.grinqh_kv_bytes(desc(g, **kw))
    assert e.value.status == status and g.grinqh_last_error()


def attend(g, d, a, cache=(P, P, P, P), batch=(P, P, P, 2, 4, 6), q=(P, 4096, 128), out=(P, 4096, 128), lse=None, ws=P,
           ws_bytes=1 << 40):
    args = [t(*v) if v is not None else None for t, v in ((g._KvCache, cache), (g._KvBatch, batch))]
    rows = [g._Rows(*v) if v is not None else None for v in (q, out)]
    ref = lambda x: ctypes.byref(x) if x is not None else None  # noqa: E731
    return g.lib.grinqh_attend(ref(d), ref(args[0]), ref(args[1]), ref(a), ref(rows[0]), ref(rows[1]), lse, ws, ws_bytes, None)


def adesc(g, **kw):
    v = dict(heads=32, type=g.GRINQH_F16, scale=0.1, window=0, sinks=0, max_rows=3, max_len=200) | kw
    return g.AttendDesc(*v.values())


@pytest.mark.parametrize("kw,status", [
    (dict(heads=0), -1), (dict(heads=33), -1), (dict(heads=8 * 8193), -1), (dict(type=2), -2), (dict(scale=0.0), -1), (dict(scale=-1.0), -1),
    (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(window=-1), -1), (dict(sinks=-1), -1),
    (dict(max_rows=0), -1), (dict(max_len=0), -1),
])
def test_attend_desc_refusals(g, kw, status):
    n = ctypes.c_size_t()
    assert g.lib.grinqh_attend_workspace_bytes(ctypes.byref(desc(g)), ctypes.byref(adesc(g, **kw)), 2, 6, ctypes.byref(n)) == status
    assert attend(g, desc(g), adesc(g, **kw)) == status


def test_a_16_bit_cache_takes_queries_of_its_type(g):
    a = adesc(g, type=g.GRINQH_BF16)
    none = (P, P, None, None)
    assert attend(g, desc(g, format=g.GRINQH_KV_F16), a, cache=none) == g.GRINQH_EUNSUPPORTED
    assert attend(g, desc(g, format=g.GRINQH_KV_BF16), adesc(g), cache=none) == g.GRINQH_EUNSUPPORTED
    assert attend(g, desc(g, format=g.GRINQH_KV_BF16), a) == g.GRINQH_EINVAL     # scales beside a 16-bit cache


@pytest.mark.parametrize("kw", [
    dict(cache=None), dict(cache=(None, P, P, P)), dict(cache=(P, P + 8, P, P)), dict(cache=(P, P, None, P)), dict(cache=(P, P, P, P + 2)),
    dict(batch=None), dict(batch=(None, P, P, 2, 4, 6)), dict(batch=(P, None, P, 2, 4, 6)), dict(batch=(P, P, P + 1, 2, 4, 6)),
    dict(batch=(P, P, P, -1, 4, 6)), dict(batch=(P, P, P, 65536, 4, 6)), dict(batch=(P, P, P, 2, 0, 6)), dict(batch=(P, P, P, 2, 4, -1)),
    dict(batch=(P, P, P, 2, 4, (1 << 24) + 1)),
    dict(q=None), dict(q=(None, 4096, 128)), dict(q=(P + 2, 4096, 128)), dict(q=(P, 4097, 128)), dict(q=(P, 4096, 132)), dict(q=(P, -4096, 128)),
    dict(out=(P, 4096, 0)), dict(out=(P, 0, 128)), dict(out=(P, 4088, 128)), dict(out=(P, 128, 512)), dict(lse=P + 1),
])
def test_attend_refusals(g, kw):
    assert attend(g, desc(g), adesc(g), **kw) == g.GRINQH_EINVAL
    assert g.grinqh_last_error()


def test_empty_batches_are_accepted_and_enqueue_nothing(g):
    for batch in ((None, None, None, 0, 0, 6), (None, None, None, 2, 0, 0)):
        assert attend(g, desc(g), adesc(g), batch=batch, q=None, out=None, ws=None, ws_bytes=0) == g.GRINQH_OK


def test_write_and_read_refusals(g):
    c, b = g._KvCache(P, P, P, P), g._KvBatch(P, P, P, 2, 4, 6)
    ok, odd, over = g._Rows(P, 1024, 128), g._Rows(P, 1027, 128), g._Rows(P, 1000, 128)
    d = desc(g)
    for f in (g.lib.grinqh_kv_write, g.lib.grinqh_kv_read):
        r = ctypes.byref
        assert f(r(d), r(c), r(b), 3, r(ok), r(ok), None) == g.GRINQH_EINVAL
        assert f(r(d), r(c), r(b), 0, r(odd), r(ok), None) == g.GRINQH_EINVAL
        assert f(r(d), r(c), r(b), 0, r(ok), None, None) == g.GRINQH_EINVAL
        assert f(None, r(c), r(b), 0, r(ok), r(ok), None) == g.GRINQH_EINVAL
        assert f(r(d), None, r(b), 0, r(ok), r(ok), None) == g.GRINQH_EINVAL
        assert f(r(d), r(c), None, 0, r(ok), r(ok), None) == g.GRINQH_EINVAL
    assert g.lib.grinqh_kv_read(r(d), r(c), r(b), 0, r(over), r(ok), None) == g.GRINQH_EINVAL   # overlapping outputs


def test_workspace_size_is_a_host_matter(g):
    n = ctypes.c_size_t()
    for B, rows, status in [(2, 6, 0), (0, 0, 0), (-1, 6, -1), (2, -1, -1)]:
        assert g.lib.grinqh_attend_workspace_bytes(ctypes.byref(desc(g)), ctypes.byref(adesc(g)), B, rows, ctypes.byref(n)) == status
    assert g.lib.grinqh_attend_workspace_bytes(ctypes.byref(desc(g)), ctypes.byref(adesc(g)), 2, 6, None) == g.GRINQH_EINVAL


def test_rows_times_heads_fit_32_bits(g):
    n, rows = ctypes.c_size_t(), 1 << 24
    for heads, status in ((64, g.GRINQH_OK), (72, g.GRINQH_ESIZE)):
        a = adesc(g, heads=heads)
        assert g.lib.grinqh_attend_workspace_bytes(ctypes.byref(desc(g)), ctypes.byref(a), 2, rows, ctypes.byref(n)) == status
    assert attend(g, desc(g), a, batch=(P, P, P, 2, 4, rows)) == g.GRINQH_ESIZE


@pytest.mark.parametrize("q", [(P, (1 << 36) + 8, 128), (P, 4096, (1 << 36) + 8)])
def test_strides_are_bounded(g, q):
    assert attend(g, desc(g), adesc(g), q=q) == g.GRINQH_EINVAL
    assert attend(g, desc(g), adesc(g), out=q) == g.GRINQH_EINVAL
