"""Calls of the cache and attention through the binding: streams, arrays that change under a handle, alignments, rows that
are not written."""
import numpy as np
import pytest

from test_gpu_kv import Case, g, self_equal, torch, up  # noqa: F401 (fixtures)

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
