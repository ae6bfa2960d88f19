"""Gates of every type, per channel and per row, against the float64 oracle: bounds of test_gpu_norm.py."""
import numpy as np
import pytest

from oracle.kv_oracle import round_to
from test_gpu_norm import Data, g, kinds, torch  # noqa: F401 (fixtures)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("gate", ["channel", "row", "one for all"])
@pytest.mark.parametrize("y,h,post,pre", [("f16", "bf16", "rms", "rms"), ("bf16", "f32", "layer", "layer"), ("f32", "f16", None, "rms"), ("f32", None, "rms", None)])
@pytest.mark.parametrize("rows,n", [(1, 1), (3, 7), (6, 333), (5, 1001), (4, 2048), (3, 4099), (2, 8190), (2, 16385)])
def test_types_of_gates(g, torch, kind, gate, y, h, post, pre, rows, n):  # noqa: F811
    if n == 1 and "layer" in (post, pre):
        post, pre = (None, "rms")      # one value less its mean is nothing
    d = Data(rows, n, y=y, h=h, post=post, pre=pre, gate="row", bias=True, scale=-0.75, seed=n)
    whole = round_to(d.rng.standard_normal((rows, n)) * 2, kind)
    if gate != "row":
        whole = np.broadcast_to(whole[:1], (rows, n)).copy()
    d.vectors["gate"] = whole
    ys, hs, vectors = d.up(torch)
    t = torch.from_numpy(whole).to(kinds(torch)[kind]).cuda()
    vectors["gate"] = {"row": t, "channel": t[0], "one for all": t[:1].expand(rows, n)}[gate]
    d.check(g.grinqh_norm(ys, hs, **vectors, **d.options(g), x_dtype=torch.float16))


@pytest.mark.parametrize("kind", ["f16", "bf16"])
def test_strides_and_alignments_of_16_bit_gates(g, torch, kind):  # noqa: F811
    """Gates that are slices of wider rows, from any element on, and a gate of infinities where y is 0: NaN there alone."""
    n = 1001
    d = Data(6, n, y="f32", h="f32", x="f32", post=None, pre=None, gate="row", seed=7)
    whole = round_to(d.vectors["gate"], kind)
    d.vectors["gate"] = whole
    ys, hs, vectors = d.up(torch)
    for before in (1, 2, 3, 5, 8):
        wide = torch.full((6, before + n + 3), float("nan"), dtype=kinds(torch)[kind], device="cuda")
        wide[:, before:before + n] = torch.from_numpy(whole).to(wide.dtype)
        d.check(g.grinqh_norm(ys, hs, **(vectors | {"gate": wide[:, before:before + n]}), **d.options(g)))
    vectors["gate"] = torch.from_numpy(whole).to(kinds(torch)[kind]).cuda()
    vectors["gate"][2, 5] = float("inf")
    ys[2, 5] = 0
    got = g.grinqh_norm(ys, hs, **vectors, **d.options(g))[0]
    assert torch.isnan(got[2, 5]) and int(torch.isnan(got).sum()) == 1
