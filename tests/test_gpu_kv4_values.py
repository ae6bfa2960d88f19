"""Attention over 4 bits where values, scores and queries lie far apart or far from one: what test_gpu_kv_values.py holds of the
other formats.  A group of one value is that as its base, with a step of zero."""
import numpy as np
import pytest

from oracle import kv_oracle as kv
from test_gpu_kv import down, forced, g, torch  # noqa: F401 (fixtures)
from test_gpu_kv4 import TYPES, Case4
from test_gpu_kv_values import U, error_and_bound

pytestmark = pytest.mark.gpu


def level(c, name, at, group, value):
    """The channels of one group of a row, all of one value."""
    c.groups[name][at + (group,)] = 0, value


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("page", [4, 16, 64])
@pytest.mark.parametrize("n,L", [(1, 100), (8, 100), (60, 100)])
def test_scores_past_the_integers_of_fp32(g, torch, forced, type, page, n, L):  # noqa: F811
    """Scores whose spacing in fp32 is many powers of two, each far from the next (up to 2^31, and of bf16 queries 2^54): every row is
    the value of its largest score.  That token's weight is a power of two, and nothing else has one."""
    c = Case4(g, torch, [(n, L)], type=type, H=1, G=2, D=64, page=page, seed=25)
    keys, query = 64.0 * c.rng.permutation(L) + 16384, 60000.0 if type == "f16" else 2.0 ** 40     # exact in fp16, scores 2^21 and more apart
    c.groups["k"][:] = 0
    for t in range(L):
        level(c, "k", (c.table[0, t // page], 0, t % page), 0, keys[t])
    c.q = np.zeros_like(c.q)
    c.q[:, 0, 0], c.q[:, 1, 0] = query, -query
    c.q = kv.round_to(c.q, type)
    c.settle().upload()
    out, lse = c.attend(scale=1.0, max_rows=n)
    ref, ref_lse, _, _ = c.want(scale=1.0)
    for i in range(n):
        seen = keys[:L - n + i + 1]
        for h, t in enumerate((seen.argmax(), seen.argmin())):
            assert np.abs(ref[i, h] - c.pool["v"][c.table[0, t // page], 0, t % page]).max() <= 1e-12
    assert (np.abs(down(out) - ref) <= (0 if type == "f16" else U[type] * np.abs(ref))).all()   # fp16 values in fp16 pass as they are
    assert (np.abs(down(lse) / ref_lse - 1) <= 2.0 ** -20).all()


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("n", [1, 8])
@pytest.mark.parametrize("nats", [13.0, 15.5, 16.5, 17.5])
def test_a_long_tail_behind_a_dominating_token(g, torch, forced, type, n, nats):  # noqa: F811
    """A first token whose values are zero stands 13 .. 17.5 nats above 8191 others, which make the whole output: a weight below 2^-14 is
    rounded in steps of 2^-24 of a reference that is 2^-9 of the largest weight and less, so 2^-34 sum |v| is what that costs a row."""
    L, D = 8192, 64
    c = Case4(g, torch, [(n, L)], type=type, H=1, G=2, D=D, page=64, seed=20)
    c.q = np.zeros_like(c.q)
    c.q[:, :, 0] = 1.0
    first = (c.table[0, 0], 0, 0)
    c.groups["k"][:] = 0
    level(c, "k", first, 0, nats)
    c.codes["v"], c.groups["v"] = kv.quantise4(c.rng.uniform(0.5, 1.5, c.codes["v"].shape))
    c.groups["v"][first] = 0
    c.settle().upload()
    out, lse = c.attend(scale=1.0, max_rows=n)
    total = np.abs(c.pool["v"])[c.table[0]].sum((0, 1, 2)).max()
    err, bound = error_and_bound(c, out, 1.0, np.full(c.rows, 2.0 ** -34 * total))
    assert (err <= bound).all(), (err / bound).max()
    assert np.abs(down(lse) - c.want(scale=1.0)[1]).max() <= 2 * D * 2.0 ** -24 * nats + 2.0 ** -20 * (1 + nats)


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("base", [2.0 ** 21, 2.0 ** 22 - 2048, 2.0 ** 23 - 2048, 2.0 ** 24 - 2048, -2.0 ** 22 - 2048, -2.0 ** 24 - 2048])
@pytest.mark.parametrize("step", [5, 14, 16])
def test_large_scores_that_rise_tile_by_tile(g, torch, forced, type, base, step):  # noqa: F811
    """Scores near the powers of two where their spacing doubles, rising with every 32 tokens: whatever the rounding of a score makes of
    its weight, outputs are averages of the values, so they lie between their bounds (within the weights' and the output's rounding)."""
    L, D, page = 1024, 64, 64
    c = Case4(g, torch, [(1, L)], type=type, H=1, G=1, D=D, page=page, seed=26)
    c.q = np.zeros_like(c.q)
    c.q[0, 0, 0], c.q[0, 0, 32] = 2048, 1
    for t in range(L):
        at = (c.table[0, t // page], 0, t % page)
        level(c, "k", at, 0, base / 2048)
        level(c, "k", at, 1, 1800 + t // 32 * step)
    c.codes["v"], c.groups["v"] = kv.quantise4(c.rng.uniform(0.5, 1.5, c.codes["v"].shape))
    c.settle().upload()
    out, lse = c.attend(scale=float(np.log(2)))
    held, far = c.pool["v"][c.table[0]], 2.0 * (U[type] + U["f16"] + 2.0 ** -12)
    assert held.min() - far <= down(out).min() and down(out).max() <= held.max() + far
    assert np.isfinite(down(lse)).all()


@pytest.mark.parametrize("power,scale", [(-120, 128 ** -0.5), (-128, 1 / 128), (-131, 1 / 128), (-80, 2.0 ** -60), (-60, 2.0 ** -149), (0, 2.0 ** -149),
                                         (100, 2.0 ** -140)])
@pytest.mark.parametrize("seqs", [[(1, 90), (40, 200), (70, 70)], [(1, 90), (4, 200), (1, 1)]])
def test_queries_whose_scores_vanish(g, torch, forced, power, scale, seqs):  # noqa: F811
    """bf16 queries, down to subnormal ones, under scales that take the scores to zero or near it: plain averages of what a row sees."""
    c = Case4(g, torch, seqs, type="bf16", H=1, G=4, page=32, seed=21)
    c.q[1:] = kv.round_bf16(c.q[1:] * 2.0 ** power)     # the first row keeps scores of its own
    c.upload()
    scale = float(np.float32(scale))
    c.check(*c.attend(scale=scale, max_rows=max(n for n, _ in seqs)), scale=scale)


@pytest.mark.parametrize("type,power,scale", [("f16", 0, 3e38), ("bf16", 0, 3e38), ("bf16", 120, 2.0 ** 30)])
@pytest.mark.parametrize("n", [4, 40])
def test_scores_of_zero_under_a_large_scale(g, torch, forced, type, power, scale, n):  # noqa: F811
    """Queries that keys of zero meet: scores of zero, whatever the scale."""
    c = Case4(g, torch, [(1, 90), (n, 200)], type=type, H=1, G=4, page=64, seed=22)
    c.q = kv.round_to(c.q * 2.0 ** power, type)
    c.groups["k"][:] = 0
    c.settle().upload()
    scale = float(np.float32(scale))
    c.check(*c.attend(scale=scale, max_rows=n), scale=scale)


@pytest.mark.parametrize("type,large", [("f16", 60000.0), ("bf16", 2.0 ** 40)])
@pytest.mark.parametrize("n,page", [(1, 64), (4, 16), (5, 4), (40, 32)])
def test_infinite_queries(g, torch, forced, type, large, n, page):  # noqa: F811
    """A channel of -inf along positive keys makes every score -inf, and the row zeros, beside finite channels of any size; one of
    +inf or NaN makes the row NaN."""
    c = Case4(g, torch, [(n, 90)], type=type, H=1, G=4, page=page, seed=23)
    c.groups["k"][..., 0, :] = np.float16(0.125), np.float16(0.5)    # the first group's values: 0.5 to 2.375
    c.q[:, 0, 0], c.q[:, 0, 1], c.q[:, 0, 2] = -np.inf, large, -large
    c.q[:, 1, 0], c.q[:, 1, 1] = np.inf, large
    c.q[:, 2, 5] = np.nan
    c.settle().upload()
    out, lse = c.attend(max_rows=n)
    got, z = down(out), down(lse)
    assert (got[:, 0] == 0).all() and (z[:, 0] == -np.inf).all()
    assert np.isnan(got[:, 1:3]).all() and np.isnan(z[:, 1:3]).all()
    c.check(out, lse)


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("n,page", [(1, 64), (8, 16), (70, 32)])
def test_values_and_keys_at_the_ends_of_their_range(g, torch, forced, type, n, page):  # noqa: F811
    """Groups from -2^15 to 2^15, and of subnormal steps and bases, as kv_write makes them of such rows."""
    c = Case4(g, torch, [(n, 150)], type=type, H=2, G=2, D=64, page=page, seed=27)
    x = {name: c.rng.uniform(-1, 1, c.codes[name].shape) for name in "kv"}
    x["k"][..., :32] *= 2.0 ** -22
    x["v"][..., :32] *= 2.0 ** 15
    x["v"][..., 32:] *= 2.0 ** -20
    for name in "kv":
        c.codes[name], c.groups[name] = kv.quantise4(x[name])
    c.settle().upload()
    out, lse = c.attend(max_rows=n)
    ref, ref_lse, weight, spread = c.want()
    # subnormal outputs of fp16 are rounded in steps of 2^-24
    err, bound = error_and_bound(c, out, None, np.full(c.rows, 2.0 ** -25))
    absent = 2.0 ** -34 * np.abs(c.pool["v"]).max((0, 1, 2)) * 150     # weights under fp16's normal range
    assert (err <= bound + absent).all(), (err / bound).max()
    d = 2 * c.D * 2.0 ** -24 * spread
    assert (np.abs(down(lse) - ref_lse) <= d + 2.0 ** -20 * (1 + np.abs(ref_lse))).all()
