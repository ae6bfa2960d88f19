"""grinqh_norm over as many rows as it takes: more workgroups, and more threads, than one axis of a grid has."""
import pytest

from test_gpu_norm import g, torch  # noqa: F401 (fixtures)

pytestmark = pytest.mark.gpu

MOST = 1 << 24


@pytest.fixture(autouse=True)
def memory_goes_back(torch):  # noqa: F811
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n", [1025, 2048, 520])
def test_rows_of_more_than_one_axis(g, torch, n):  # noqa: F811
    """Where a second axis begins: the rows about its start, the last ones and a sample are those of a call of their own, bit for bit."""
    rows = (1 << 20) * (4 if n < 1024 else 1) + 5
    h = torch.empty((rows, n), dtype=torch.bfloat16, device="cuda")
    for part in h.split(1 << 18):
        part.normal_()
    x = torch.full((rows + 1, n), 777.0, dtype=torch.float16, device="cuda")
    g.grinqh_norm(None, h, x=x[:rows])
    assert (x[rows] == 777).all()
    some = torch.cat([torch.arange(0, 9), torch.randint(rows, (400,)), torch.arange(rows // 2 - 20, rows // 2 + 20),
                      torch.arange(rows - 40, rows)]).cuda()
    assert torch.equal(g.grinqh_norm(None, h[some])[1], x[some])
    for part in x[:rows].split(1 << 18):    # and none is left out
        assert ((part.float() ** 2).mean(-1) - 1).abs().max() < 0.01   # fp16's roundings


@pytest.mark.parametrize("n,rows", [(1025, MOST), (1, MOST), (4097, 1 << 23)])
def test_the_most_rows(g, torch, n, rows):  # noqa: F811
    """One row for all (stride 0), written to each of them."""
    h = torch.randn((1, n), device="cuda")
    want = g.grinqh_norm(None, h)[1]
    x = torch.full((rows, n), 777.0, dtype=torch.float16, device="cuda")
    g.grinqh_norm(None, h.expand(rows, n), x=x)
    for part in x.split(1 << 19):
        assert (part == want).all()
