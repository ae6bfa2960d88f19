"""grinqh_norm where a row's values lie close together, far from zero, against the float64 oracle.

The kernel takes the mean off twice: a rounded one, m, then the mean r of what that leaves, (v - m) - r.  With u = 2^-24, S = 56 u of a
sum's terms and F = 32 u of a factor (test_gpu_norm.py):
  equal values   m is off by at most 53 u of a value (31 additions in a lane, 6 exchanges, 15 waves, the product by 1 / n), so by d = k ulp
                 with k <= 106, wherever m lies; v - m is exact (values within a factor of two of each other), n d is less than
                 2^15 107 < 2^22 ulp, so every partial sum of it is exact, and r = n d / n is d: what is left is 0, not something small
  others         v - m is rounded, by u of itself, and less r again; r is off by (S + u) mean|v - m| and u |r|.  |v - m| is at most |c| + D
                 with c the centred value and D = 53 u |mean|, the bound of m's error; so c is off by e = 3 u (|c| + D) + (S + 2 u) (mean|c| + D),
                 x by factor (e + |x| ||e||), as the relative error of the factor is that of c in the two-norm, and by F |x|."""
import numpy as np
import pytest

from oracle import step_oracle as step
from test_gpu_norm import S, U, F, g, torch  # noqa: F401 (fixtures)

pytestmark = pytest.mark.gpu

WIDTHS = [1, 2, 3, 7, 41, 100, 513, 777, 1001, 2047, 4096, 5001, 12289, 16385, 32768]
ALIKE = [0.1, 1000.3, -7.7e8, 30000.0, 1e-3, 3.3e-12, 0.0]


def both(g, t, eps, **kw):  # noqa: F811
    """x of the pre norm and of the post norm of rows t."""
    yield g.grinqh_norm(None, t, pre=g.GRINQH_NORM_LAYER, eps=eps, x_dtype=t.dtype, **kw)[1]
    yield g.grinqh_norm(t, None, pre=g.GRINQH_NORM_NONE, post=g.GRINQH_NORM_LAYER, eps=eps, **{"post_" + k: v for k, v in kw.items()})[0]


@pytest.mark.parametrize("n", WIDTHS)
@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_equal_values_leave_nothing(g, torch, n, kind):  # noqa: F811
    """A row of one value is its bias, and with eps = 0 NaN."""
    t = torch.tensor(ALIKE, device="cuda").to(getattr(torch, kind))[:, None].expand(len(ALIKE), n).contiguous()
    weight, bias = torch.randn(n, device="cuda"), torch.randn(n, device="cuda")
    for eps in (1e-5, 1e-20, 1e-28):
        for x in both(g, t, eps):
            assert (x == 0).all()
        for x in both(g, t, eps, weight=weight, bias=bias):
            assert torch.equal(x, bias.to(x.dtype).expand_as(x))
    for x in both(g, t, 0.0):
        assert torch.isnan(x).all()


@pytest.mark.parametrize("n", [41, 777, 2047, 4096, 5001, 32768])
@pytest.mark.parametrize("apart", [1e4, 1e6, 3e7])
@pytest.mark.parametrize("eps", [0.0, 1e-5])
def test_values_close_together_far_from_zero(g, torch, n, apart, eps):  # noqa: F811
    """Means of 1e4 to 3e7 standard deviations (there the values are a few steps of fp32 apart); one row has a channel far outside."""
    rng = np.random.default_rng(n)
    v = np.float32(apart + rng.standard_normal((4, n)))
    v[1] *= -1
    v[2, n // 2] = 3 * apart
    v[3] = np.float32(apart) * (1 + np.float32(2.0 ** -22) * (np.arange(n) == n - 1))
    t, ref = torch.from_numpy(v).cuda(), v.astype(np.float64)
    eps = float(np.float32(eps))
    c = ref - ref.mean(-1, keepdims=True)
    factor = 1 / np.sqrt((c * c).mean(-1, keepdims=True) + eps)
    want = c * factor
    D = 53 * U * np.abs(ref).mean(-1, keepdims=True)
    e = 3 * U * (np.abs(c) + D) + (S + 2 * U) * (np.abs(c).mean(-1, keepdims=True) + D)
    whole = np.sqrt((e * e).mean(-1, keepdims=True)) * factor
    bound = factor * e + np.abs(want) * (whole + F) + U
    for x in both(g, t, eps):
        far = np.abs(x.cpu().double().numpy() - want) - bound
        assert (far <= 0).all(), (far.max(), np.unravel_index(far.argmax(), far.shape))
    assert np.abs(want - step.norm(None, ref, pre="layer", eps=eps)[1]).max() <= 1e-6   # the oracle's mean in float64 does as well


@pytest.mark.parametrize("n", [1, 41, 777, 4096, 5001, 16385])
@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("eps", [1e-5, 1e-32, 1e-38, 1e-44, 3e38])
def test_equal_values_of_any_size_leave_nothing(g, torch, n, kind, eps):  # noqa: F811
    """eps > 0: the root is that of eps, however far below the values' square it lies."""
    sizes = [0.0, 2.0 ** -149, -1e-40, 2.0 ** -60, 1.7e-20, -2.0 ** 65, 1.3e20, 2.0 ** 125, -2.0 ** 125, 3e38, 5.0]
    t = torch.tensor(sizes, device="cuda").to(getattr(torch, kind))[:, None].expand(len(sizes), n).contiguous()
    weight, bias = torch.randn(n, device="cuda"), torch.randn(n, device="cuda")
    for x in both(g, t, eps):
        assert (x == 0).all(), sizes[int((x != 0).any(-1).nonzero()[0])]
    for x in both(g, t, eps, weight=weight, bias=bias):
        assert torch.equal(x, bias.to(x.dtype).expand_as(x))


@pytest.mark.parametrize("size,eps", [(2.0 ** -60, 1e-32), (1e-38, 1e-32), (1e-42, 1e-32), (1e-38, 1e-44), (1e-20, 1e-38), (1e30, 1e-38), (3e37, 3e38), (1e19, 3e38)])
@pytest.mark.parametrize("n", [41, 5001])
def test_small_and_large_eps(g, torch, size, eps, n):  # noqa: F811
    """eps beside squares that leave fp32's range: rows of x in fp32, down to its subnormal numbers."""
    rng = np.random.default_rng(n)
    v = (rng.uniform(-1, 1, (3, n)) * size).astype(np.float32)
    t, ref, eps = torch.from_numpy(v).cuda(), v.astype(np.float64), float(np.float32(eps))
    for kind, name in ((g.GRINQH_NORM_RMS, "rms"), (g.GRINQH_NORM_LAYER, "layer")):
        x = g.grinqh_norm(None, t, pre=kind, eps=eps, x_dtype=torch.float32)[1].cpu().double().numpy()
        want = step.norm(None, ref, pre=name, eps=eps)[1]
        # a centred value is off by a step of the values' mean, at least 2^-149 (and as much when the row is scaled), x by factor times that
        c = ref - ref.mean(-1, keepdims=True) if name == "layer" else ref
        factor = 1 / np.sqrt((c * c).mean(-1, keepdims=True) + eps)
        e = (S + 4 * U) * np.abs(ref).mean(-1, keepdims=True) + 3 * U * np.abs(c) + 2.0 ** -147 if name == "layer" else 0.0
        whole = np.sqrt((e * e).mean(-1, keepdims=True)) * factor if name == "layer" else 0.0
        assert (np.abs(x - want) <= factor * e + np.abs(want) * (F + whole) + 2.0 ** -149).all()
