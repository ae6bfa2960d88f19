"""Attention over the cache where values, scores and queries lie far apart or far from one, against the float64 oracle.

Bounds are those of test_gpu_kv.py, with its last term, for weights under fp16's normal range, as the case needs it."""
import numpy as np
import pytest

from oracle import kv_oracle as kv
from test_gpu_kv import FORMATS, Case, down, forced, g, torch  # noqa: F401 (fixtures)

pytestmark = pytest.mark.gpu

U = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def error_and_bound(c, out, scale, absent):
    """|out - ref| and its bound; absent [rows]: what a row's weights below the normal range may cost."""
    ref, _, weight, spread = c.want(scale=scale)
    d = 2 * c.D * 2.0 ** -24 * spread[..., None]
    bound = U[c.type] * np.abs(ref) + (U["bf16" if c.fmt == "bf16" else "f16"] + 2 * d + 2.0 ** -14) * weight
    return np.abs(down(out) - ref), bound + absent[:, None, None]


@pytest.mark.parametrize("fmt,type", FORMATS)
@pytest.mark.parametrize("n,L", [(1, 100), (60, 100)])
def test_scores_past_the_integers_of_fp32(g, torch, forced, fmt, type, n, L):  # noqa: F811
    """Scores whose spacing in fp32 is many powers of two, each far from the next (fp16 up to 2^31, else up to 2^106): every
    row is the value of its largest score.  That token's weight is a power of two, 1 in fp32 but for what the others add."""
    c = Case(g, torch, [(n, L)], fmt=fmt, type=type, H=1, G=2, D=64, page=16, seed=25)
    order = c.rng.permutation(L)
    if fmt == "f16":
        keys, query = 64.0 * order + 16384, 60000.0     # exact in fp16; scores more than 2^21 apart
    else:
        keys, query = 2.0 ** (order // 2 + 3) * np.where(order % 2, 1.5, 1.0), 2.0 ** (40 if type == "bf16" else 10)
    k = np.zeros((c.n_pages, 1, 16, 64))
    for t in range(L):
        k[c.table[0, t // 16], 0, t % 16, 0] = keys[t]
    c.q = np.zeros_like(c.q)
    c.q[:, 0, 0], c.q[:, 1, 0] = query, -query
    c.q = kv.round_to(c.q, type)
    if fmt == "i8":
        c.pool["k"], c.scales["k"] = kv.quantise(k)
    else:
        c.pool["k"] = kv.round_to(k, fmt)
    c.upload()
    out, lse = c.attend(scale=1.0)
    ref, ref_lse, _, _ = c.want(scale=1.0)
    tokens = np.arange(L)
    for i in range(n):
        seen = keys[:L - n + i + 1]
        for h, t in enumerate((seen.argmax(), seen.argmin())):
            v = kv.values(c.pool["v"], c.scales["v"])[c.table[0, tokens[t] // 16], 0, tokens[t] % 16]
            assert np.abs(ref[i, h] - v).max() <= 1e-12
    # 16-bit values pass as they are; at 8 bits their scale is rounded to fp16 and the product to the output's type
    bound = 0 if fmt != "i8" else (U[type] + 2.0 ** -11 + 2.0 ** -20) * np.abs(ref)
    assert (np.abs(down(out) - ref) <= bound).all()
    assert (np.abs(down(lse) / ref_lse - 1) <= 2.0 ** -20).all()


@pytest.mark.parametrize("fmt", ["f16", "bf16", "i8"])
@pytest.mark.parametrize("nats", [13.0, 15.5, 16.5, 17.5])
def test_a_long_tail_behind_a_dominating_token(g, torch, forced, fmt, nats):  # noqa: F811
    """A first token whose values are zero stands 13 .. 17.5 nats above 8191 others, which make the whole output.

    A weight is rounded to 16 bits once.  It is at most 2^6 against the row's reference, and the largest is at least 1 of it.
    Lifted by 2^9 it stays below fp16's 2^16, so that below 2^-14 it is rounded in steps of 2^-24, an error of
    2^-25 2^-9 of the largest weight and less of the sum: 2^-34 sum |v| over the row's tokens.  (At 8 bits it is the weight times
    its scale over the power of two above the largest scale that is rounded: at most twice 2^-34 of the largest value.)"""
    L, D = 8192, 64
    type = "bf16" if fmt == "bf16" else "f16"
    c = Case(g, torch, [(1, L)], fmt=fmt, H=1, G=2, D=D, page=64, type=type, seed=20)
    c.q = np.zeros_like(c.q)
    c.q[:, :, 0] = 1.0
    first = (c.table[0, 0], 0, 0)
    for name, x in (("k", np.zeros((c.n_pages, 1, 64, D))), ("v", c.rng.uniform(0.5, 1.5, (c.n_pages, 1, 64, D)))):
        if name == "k":
            x[first + (0,)] = nats
        else:
            x[first] = 0
        if fmt == "i8":
            c.pool[name], c.scales[name] = kv.quantise(x)
        else:
            c.pool[name] = kv.round_to(x, fmt)
    c.upload()
    out, lse = c.attend(scale=1.0)
    v = np.abs(kv.values(c.pool["v"], c.scales["v"]))
    total = v[c.table[0]].sum((0, 1, 2)).max() if fmt != "i8" else 2 * L * v.max()
    err, bound = error_and_bound(c, out, 1.0, np.full(c.rows, 2.0 ** -34 * total))
    assert (err <= bound).all(), (err / bound).max()
    ref = c.want(scale=1.0)[1]
    assert np.abs(down(lse) - ref).max() <= 2 * D * 2.0 ** -24 * nats + 2.0 ** -20 * (1 + nats)


@pytest.mark.parametrize("fmt", ["f16", "bf16", "i8"])
@pytest.mark.parametrize("base", [2.0 ** 21, 2.0 ** 22 - 2048, 2.0 ** 23 - 2048, 2.0 ** 24 - 2048, -2.0 ** 22 - 2048, -2.0 ** 24 - 2048])
@pytest.mark.parametrize("step", [5, 14, 16])
def test_large_scores_that_rise_tile_by_tile(g, torch, forced, fmt, base, step):  # noqa: F811
    """Scores near the powers of two where their spacing doubles, rising with every 32 tokens: whatever the rounding of a score makes of
    its weight, outputs are averages of the values, so they lie between their bounds (within the weights' and the output's
    rounding)."""
    L, D = 1024, 64
    type = "bf16" if fmt == "bf16" else "f16"
    c = Case(g, torch, [(1, L)], fmt=fmt, H=1, G=1, D=D, page=64, type=type, seed=26)
    c.q = np.zeros_like(c.q)
    c.q[0, 0, :2] = 2048, 1
    k, v = np.zeros((c.n_pages, 1, 64, D)), c.rng.uniform(0.5, 1.5, (c.n_pages, 1, 64, D))
    for t in range(L):
        k[c.table[0, t // 64], 0, t % 64, :2] = base / 2048, 1800 + t // 32 * step
    for name, x in (("k", k), ("v", v)):
        if fmt == "i8":
            c.pool[name], c.scales[name] = kv.quantise(x)
        else:
            c.pool[name] = kv.round_to(x, fmt)
    c.upload()
    out, lse = c.attend(scale=float(np.log(2)))
    held, far = kv.values(c.pool["v"], c.scales["v"])[c.table[0]], 2.0 * (U[type] + U["bf16" if fmt == "bf16" else "f16"] + 2.0 ** -12)
    assert held.min() - far <= down(out).min() and down(out).max() <= held.max() + far
    assert np.isfinite(down(lse)).all()


@pytest.mark.parametrize("power,scale", [(-120, 128 ** -0.5), (-128, 1 / 128), (-131, 1 / 128), (-80, 2.0 ** -60), (-60, 2.0 ** -149), (0, 2.0 ** -149),
                                         (100, 2.0 ** -140)])
def test_queries_whose_scores_vanish(g, torch, forced, power, scale):  # noqa: F811
    """bf16 queries against an 8-bit cache, down to subnormal ones, under scales that take the scores to zero or near it:
    plain averages of what a row sees."""
    c = Case(g, torch, [(1, 90), (40, 200), (70, 70)], type="bf16", H=1, G=4, page=16, seed=21)
    c.q[1:] = kv.round_bf16(c.q[1:] * 2.0 ** power)     # the first row keeps scores of its own
    c.upload()
    scale = float(np.float32(scale))
    c.check(*c.attend(scale=scale), scale=scale)


@pytest.mark.parametrize("fmt,type,power,scale", [("f16", "f16", 0, 3e38), ("bf16", "bf16", 0, 3e38), ("i8", "f16", 0, 3e38), ("i8", "bf16", 120, 2.0 ** 30)])
def test_scores_of_zero_under_a_large_scale(g, torch, forced, fmt, type, power, scale):  # noqa: F811
    """Queries that keys of zero meet: scores of zero, whatever the scale."""
    c = Case(g, torch, [(1, 90), (40, 200)], fmt=fmt, type=type, H=1, G=4, page=16, seed=22)
    c.q = kv.round_to(c.q * 2.0 ** power, type)
    c.pool["k"] = np.zeros_like(c.pool["k"])
    if fmt == "i8":
        c.scales["k"] = np.zeros_like(c.scales["k"])
    c.upload()
    scale = float(np.float32(scale))
    c.check(*c.attend(scale=scale), scale=scale)


def test_infinite_queries(g, torch, forced):  # noqa: F811
    """A channel of -inf along positive keys makes every score -inf, and the row zeros, beside finite channels far outside
    fp16's range; one of +inf or NaN makes the row NaN."""
    c = Case(g, torch, [(5, 90)], type="bf16", H=1, G=4, page=16, seed=23)
    c.pool["k"][..., 0] = np.maximum(np.abs(c.pool["k"][..., 0].astype(int)), 1)
    c.q[:, 0, 0], c.q[:, 0, 1], c.q[:, 0, 2] = -np.inf, 2.0 ** 40, -2.0 ** 40
    c.q[:, 1, 0], c.q[:, 1, 1] = np.inf, 2.0 ** 40
    c.q[:, 2, 5] = np.nan
    c.upload()
    out, lse = c.attend()
    got, z = down(out), down(lse)
    assert (got[:, 0] == 0).all() and (z[:, 0] == -np.inf).all()
    assert np.isnan(got[:, 1:3]).all() and np.isnan(z[:, 1:3]).all()
    c.check(out, lse)


@pytest.mark.parametrize("power", [60, 90])
def test_rows_of_a_chunk_whose_values_lie_far_apart(g, torch, forced, power):  # noqa: F811
    """8-bit values of 2^-power up to the middle of a chunk and of 2^power from there: rows before it are as exact as if
    the later tokens were not there."""
    n, L, t0 = 70, 200, 158
    c = Case(g, torch, [(n, L)], type="bf16", H=1, G=4, page=16, seed=24)
    for t in range(L):
        c.scales["v"][c.table[0, t // 16], :, t % 16] *= np.float32(2.0 ** (power if t >= t0 else -power))
    c.upload()
    out, _ = c.attend()
    top = np.abs(kv.values(c.pool["v"], c.scales["v"]))[c.table[0, :(L + 15) // 16]].max((1, 3)).reshape(-1)
    seen = np.maximum.accumulate(top)[np.arange(L - n, L)]
    err, bound = error_and_bound(c, out, None, 2.0 ** -23 * seen)
    assert (err <= bound).all(), (err / bound).max()


def test_the_smallest_values_of_a_long_sequence(g, torch):  # noqa: F811
    """11 * 2^20 tokens, all but the first page 2^5 times the first's weight, of values 2^-101 throughout: the sum of the weights and
    the values' scale both stay within fp32, their quotient would not."""
    L, page, D = 11 << 20, 64, 64
    desc = g.make_kv_desc(g.GRINQH_KV_I8, 1, D, page, 2)
    cache = g.kv_cache(desc)
    cache.k[1, 0, :, 0], cache.v[:] = 127, 64
    cache.k_scale[:], cache.v_scale[:] = 1 / 127, 2.0 ** -107
    table = torch.ones((1, L // page), dtype=torch.int32, device="cuda")
    table[0, 0] = 0
    batch = g.KvBatch(table, torch.tensor([L], dtype=torch.int32, device="cuda"), torch.tensor([0, 1], dtype=torch.int32, device="cuda"))
    q = torch.zeros((1, 1, D), dtype=torch.bfloat16, device="cuda")
    q[0, 0, 0] = 1
    g.grinqh_set_option(g.GRINQH_OPT_ATTEND_KERNEL, g.GRINQH_ATTEND_TILE)
    g.grinqh_set_option(g.GRINQH_OPT_ATTEND_SPLITS, 1)
    try:
        out = g.grinqh_attend(desc, cache, batch, q, scale=5 * float(np.log(2)))
    finally:
        g.grinqh_set_option(g.GRINQH_OPT_ATTEND_KERNEL, 0)
        g.grinqh_set_option(g.GRINQH_OPT_ATTEND_SPLITS, 0)
    # the output's rounding, the weights', that of exp and of the scores, and the sum's: additions of 2^10 to at most 2^28.5 a
    # half wave, exact while the weights are 2^5 (1 +- 2^-20) and else at most 2^-18 of it each
    bound = 2.0 ** -8 + 2.0 ** -11 + 2.0 ** -14 + 2.0 ** -10
    assert np.abs(down(out) / 2.0 ** -101 - 1).max() <= bound
