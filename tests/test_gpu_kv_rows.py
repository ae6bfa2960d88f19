"""grinqh_kv_write over as many rows as it takes."""
import pytest

from test_gpu_kv import g, torch  # noqa: F401 (fixtures)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,rows", [(64, 1 << 24), (3, 1 << 24), (200, (1 << 22) + 3)])
def test_the_most_rows(g, torch, heads, rows):  # noqa: F811
    """Rows that are one row (stride 0) of one sequence whose pages before the last two were given back: a grid of a
    row each would have more threads than an axis of it can."""
    D, page = 128, 64
    desc = g.make_kv_desc(g.GRINQH_KV_F16, heads, D, page, 3)
    cache = g.kv_cache(desc)
    width = -(-rows // page)
    table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    table[0, -2:] = torch.tensor([2, 0], dtype=torch.int32)
    batch = g.KvBatch(table, torch.tensor([rows], dtype=torch.int32, device="cuda"), torch.tensor([0, rows], dtype=torch.int32, device="cuda"))
    x = {n: torch.randn((1, heads, D), device="cuda").half() for n in "kv"}
    g.grinqh_kv_write(desc, cache, batch, *[x[n].expand(rows, heads, D) for n in "kv"])
    left = rows - (width - 1) * page
    for n in "kv":
        want = torch.zeros((3, heads, page, D), dtype=torch.float16, device="cuda")
        want[2] = x[n][0][:, None]
        want[0, :, :left] = x[n][0][:, None]
        assert torch.equal(getattr(cache, n), want)
