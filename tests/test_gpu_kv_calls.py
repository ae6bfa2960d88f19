"""Calls of the cache and attention through the binding: streams, arrays that change under a handle, alignments, rows that
are not written."""
import numpy as np
import pytest

from oracle import kv_oracle as kv
from test_gpu_kv import Case, down, forced, g, rows_of, self_equal, torch, up  # noqa: F401 (fixtures)

pytestmark = pytest.mark.gpu


def test_memory_still_in_use_on_the_current_stream(g, torch):  # noqa: F811
    """Blocks freed on the current stream, whose last kernels there have not run yet, are not what a call on another stream
    gets for its outputs and workspace."""
    c = Case(g, torch, [(1, 9000), (1, 400)], H=2, page=32).upload()
    q = up(torch, c.q, "f16")
    want = c.attend(lse=False)[0]
    rows = g.grinqh_kv_read(c.desc, c.cache, c.batch, c.rows)
    size = g.grinqh_attend_workspace_bytes(c.desc, c.heads, c.B, c.rows, max_rows=c.rows, max_len=c.width * c.page)
    assert size > 0
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    for _ in range(4):
        freed = [torch.empty_like(q), torch.empty(size, dtype=torch.uint8, device="cuda"), *[torch.empty_like(x) for x in rows]]
        torch.cuda._sleep(20_000_000)          # about 10 ms, then the blocks are overwritten
        for t in freed:
            t.fill_(255 if t.dtype == torch.uint8 else float("nan"))
        del t, freed
        out = g.grinqh_attend(c.desc, c.cache, c.batch, q, stream=side)
        k, v = g.grinqh_kv_read(c.desc, c.cache, c.batch, c.rows, stream=side)
        torch.cuda.synchronize()
        assert self_equal(torch, out, want)
        assert self_equal(torch, k, rows[0]) and self_equal(torch, v, rows[1])


def test_arrays_of_another_type_under_a_handle(g, torch):  # noqa: F811
    """A handle's checked arguments are not used again for arrays that have changed their type in place."""
    c = Case(g, torch, [(4, 9)], fmt="f16", page=16).upload()
    q = up(torch, c.q, "f16")
    g.grinqh_attend(c.desc, c.cache, c.batch, q)
    c.cache.v.data = c.cache.v.data.view(torch.bfloat16)
    with pytest.raises(TypeError):
        g.grinqh_attend(c.desc, c.cache, c.batch, q)
    c.cache.v.data = c.cache.v.data.view(torch.float16)
    g.grinqh_attend(c.desc, c.cache, c.batch, q)
    c.batch.seq_lens.data = c.batch.seq_lens.data.view(torch.float32)
    with pytest.raises(TypeError):
        g.grinqh_attend(c.desc, c.cache, c.batch, q)


@pytest.mark.parametrize("page", [8, 64])
@pytest.mark.parametrize("type", ["f16", "bf16"])
def test_scales_aligned_to_four_bytes(g, torch, forced, type, page):  # noqa: F811
    """The scales of an 8-bit cache start one word into their memory, as an allocator's slices may."""
    c = Case(g, torch, [(1, 77), (40, 300), (90, 90)], type=type, H=3, G=2, page=page, seed=30).upload()

    def moved(t):
        wide = torch.full((t.numel() + 2,), 5.0, device="cuda")
        wide[1:-1] = t.view(-1)
        assert wide[1:-1].data_ptr() % 16 == 4
        return wide[1:-1].view(t.shape)

    c.cache = c.cache._replace(k_scale=moved(c.cache.k_scale), v_scale=moved(c.cache.v_scale))
    c.check(*c.attend())
    x = {n: rows_of(torch, np.random.default_rng(31), c.rows, 3, 128, type, "plain") for n in "kv"}
    g.grinqh_kv_write(c.desc, c.cache, c.batch, x["k"][1], x["v"][1])
    got = g.grinqh_kv_read(c.desc, c.cache, c.batch, c.rows, dtype=torch.float32)
    for n, t in zip("kv", got):
        kv.write(c.pool[n], c.scales[n], "i8", c.table, c.lens, c.offsets, x[n][0])
        ref, _ = kv.read(c.pool[n], c.scales[n], c.table, c.lens, c.offsets, c.rows)
        assert np.array_equal(down(t), ref.astype(np.float32).astype(np.float64))
        assert np.array_equal(down(getattr(c.cache, n + "_scale")), c.scales[n].astype(np.float64))


@pytest.mark.parametrize("fmt", ["i8", "f16", "bf16"])
@pytest.mark.parametrize("offsets,lens", [
    ([2, 5, 7], [6, 9]),                    # two rows before the first sequence, two behind the last
    ([0, 0, 3, 3, 3, 9], [4, 11, 2, 0, 8]),  # sequences of no rows at either end of others
    ([9, 9, 9], [6, 9]),
    ([-4, 3, 100], [6, 12]),                # clamped to the rows
    ([5, 5, 8, 8], [3, 7, 10]),
])
def test_only_the_rows_of_sequences_are_written(g, torch, fmt, offsets, lens):  # noqa: F811
    """The whole cache after a write of new values, bit for bit, and rows read back beside rows that are left as they were."""
    rows, H, D = 9, 2, 64
    c = Case(g, torch, [(0, 12)] * len(lens), fmt=fmt, H=H, G=1, D=D, page=4, seed=32)
    c.offsets, c.lens, c.rows = np.array(offsets, np.int32), np.array(lens, np.int32), rows
    c.upload()
    rng = np.random.default_rng(33)
    x = {n: rows_of(torch, rng, rows, H, D, "f16", "plain", 2.0) for n in "kv"}
    g.grinqh_kv_write(c.desc, c.cache, c.batch, x["k"][1], x["v"][1])
    for n in "kv":
        before = c.pool[n].copy()
        kv.write(c.pool[n], c.scales[n], fmt, c.table, c.lens, c.offsets, x[n][0])
        assert np.array_equal(down(getattr(c.cache, n)), c.pool[n].astype(np.float64))
        if fmt == "i8":
            assert np.array_equal(down(getattr(c.cache, n + "_scale")), c.scales[n].astype(np.float64))
        taken = sum(min(k, L) for _, k, L in kv.sequences(c.offsets, c.lens, c.width, c.page, rows))
        assert (before != c.pool[n]).any((1, 3)).sum() == taken
    k = torch.full((rows, H, D), 5.0, device="cuda")
    v = k.clone()
    g.grinqh_kv_read(c.desc, c.cache, c.batch, rows, dtype=torch.float32, k=k, v=v)
    for n, t in (("k", k), ("v", v)):
        ref, written = kv.read(c.pool[n], c.scales[n], c.table, c.lens, c.offsets, rows)
        assert np.array_equal(down(t)[written], ref[written].astype(np.float32).astype(np.float64)) and (down(t)[~written] == 5).all()
