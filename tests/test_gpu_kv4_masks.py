"""Masks of the attention over 4 bits in every form of its kernels: pages of each class (smaller than 16 tokens, 16, 32 and more), one block
of 16 rows a wave and two, the kernel of chunks; windows and sinks that end inside tiles, pages given back, what is not
finite where rows do not see it.  Bounds are those of test_gpu_kv.py."""
import numpy as np
import pytest

from oracle import kv_oracle as kv
from test_gpu_kv import down, forced, g, torch  # noqa: F401 (fixtures)
from test_gpu_kv4 import TYPES, Case4

pytestmark = pytest.mark.gpu

PAGES = [4, 16, 32, 64, 128]
ODD = [(0.0, np.nan), (60000.0, 3.0), (np.inf, -np.inf)]


def give_back(c, seqs, window, sinks):
    """The pages that no row of a sequence sees are no longer its own."""
    for b, (n, L) in enumerate(seqs):
        first = max(0, L - n - window + 1) // c.page if window else 0
        kept = -(-sinks // c.page)
        c.table[b, min(first, kept):first] = [-1, 1 << 30][b & 1]


@pytest.mark.parametrize("page", PAGES)
@pytest.mark.parametrize("D,H,G,type", [(128, 2, 4, "f16"), (128, 1, 8, "bf16"), (64, 3, 7, "f16"), (64, 2, 1, "bf16")])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (1, 1), (33, 5), (50, 70), (100, 33)])
def test_single_rows(g, torch, forced, page, D, H, G, type, window, sinks):  # noqa: F811
    """A step of decoding: one row a sequence, lengths about the ends of tiles and pages."""
    seqs = [(1, L) for L in (1, 31, 32, 33, 64, 65, 129, 300, 513)] + [(0, 40), (1, 0)]
    c = Case4(g, torch, seqs, type=type, D=D, H=H, G=G, page=page, fill=ODD[page % 3], seed=page)
    give_back(c, seqs, window, sinks)
    c.upload()
    c.check(*c.attend(window=window, sinks=sinks, max_rows=1, max_len=513), window, sinks)


@pytest.mark.parametrize("page", PAGES)
@pytest.mark.parametrize("n,G", [(2, 8), (4, 4), (3, 5), (16, 1), (4, 8), (17, 1), (8, 4)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3), (45, 40)])
def test_a_few_rows(g, torch, forced, page, n, G, window, sinks):  # noqa: F811
    """Drafts: 15 to 32 rows of a kv head, one block of 16 rows a wave or two."""
    seqs = [(n, L) for L in (n, 47, 64, 200, 333)] + [(1, 90)]
    type = TYPES[G % 2]
    c = Case4(g, torch, seqs, type=type, D=[64, 128][n % 2], H=2, G=G, page=page, fill=ODD[n % 3], seed=n)
    give_back(c, seqs, window, sinks)
    c.upload()
    c.check(*c.attend(window=window, sinks=sinks, max_rows=n, max_len=333), window, sinks)


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("D,G,page", [(128, 4, 32), (64, 3, 64), (128, 2, 64), (64, 2, 32), (128, 3, 128)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 5), (130, 70)])
@pytest.mark.parametrize("fill", ODD)
def test_chunks(g, torch, forced, type, D, G, page, window, sinks, fill):  # noqa: F811
    seqs = [(1, 1), (90, 300), (0, 3), (1, 500), (9, 4), (64, 64)]
    c = Case4(g, torch, seqs, type=type, D=D, H=2, G=G, page=page, fill=fill)
    give_back(c, seqs, window, sinks)
    c.upload()
    c.check(*c.attend(window=window, sinks=sinks, max_rows=90, max_len=500), window, sinks)


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("page", [32, 64])
@pytest.mark.parametrize("n,G", [(100, 2), (3, 4), (8, 2), (7, 4)])
def test_masked_groups_that_are_not_finite(g, torch, forced, type, page, n, G):  # noqa: F811
    """One token with groups of NaN and past fp16's range: it reaches the rows that see it, and their channels of that group, alone."""
    L, window, D = 130, 40, 128
    for t in (L - n - window + 1, L - n - window + 2, 64, 99, L - 2, L - 1):
        if t < 0:
            continue
        c = Case4(g, torch, [(n, L)], type=type, H=1, G=G, D=D, page=page, seed=5)
        at = (c.table[0, t // page], 0, t % page)
        c.groups["v"][at + (0,)] = 0, np.nan
        c.groups["v"][at + (2,)] = 30000, 30000
        c.groups["v"][at + (3,)] = 3, -np.inf
        c.codes["v"][at] |= 8
        c.settle().upload()
        got = down(c.attend(window=window, max_rows=n)[0])
        seen = kv.sees(np.arange(L - n, L), t, window, 0)
        assert np.isfinite(got[~seen]).all()
        assert np.isnan(got[seen][..., :32]).all() and np.isfinite(got[seen][..., 32:64]).all()
        assert (got[seen][..., 64:96] == np.inf).all() and (got[seen][..., 96:] == -np.inf).all()


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("page", [4, 16, 32, 64])
@pytest.mark.parametrize("n,G", [(70, 2), (4, 4), (5, 6)])
def test_pages_out_of_range(g, torch, forced, type, page, n, G):  # noqa: F811
    """A row that sees a token of such a page is NaN, the others know nothing of it."""
    L, window = 200, 64
    c = Case4(g, torch, [(n, L), (1, 40), (1, 70)], type=type, H=2, G=G, page=page, seed=6)
    lost = (L - n - 64 + n // 2) // page    # the first rows see its end, the last ones do not
    c.table[0, lost] = -7
    c.table[1, 0] = c.n_pages
    c.upload()
    out, lse = c.attend(window=window, max_rows=n)
    c.check(out, lse, window)
    got = np.isnan(down(out))
    assert got[n].all() and not got[n + 1].any() and got[0].all()


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("page", [32, 64, 128])
@pytest.mark.parametrize("n", [1, 8, 60])
def test_a_row_depends_on_what_it_sees_alone(g, torch, forced, type, page, n):  # noqa: F811
    """The same bits whatever stands in the places that a row does not see, and in other sequences' pages."""
    outs = []
    for fill in ((1.0, 0.0), (np.nan, np.nan), (60000.0, 60000.0)):
        c = Case4(g, torch, [(min(n, 1), 77), (n, 220)], H=2, G=3, D=128, type=type, page=page, seed=11, fill=fill)
        c.upload()
        outs.append([t.cpu().view(torch.uint8).numpy() if t.dtype != torch.bfloat16 else t.cpu().view(torch.int16).numpy()
                     for t in c.attend(window=30, sinks=3, max_rows=n)])
    for o in outs[1:]:
        assert all(np.array_equal(x, y) for x, y in zip(o, outs[0]))
