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
