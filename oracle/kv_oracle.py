"""The key/value cache and the attention over it in plain numpy, 64 bits: what the library's cache entry points are
compared with.  Written from the definitions in include/grinqh.h; shares nothing with the library."""
from __future__ import annotations

import numpy as np

F16, BF16, F32 = "f16", "bf16", "f32"
KV_F16, KV_BF16, KV_I8 = "f16", "bf16", "i8"


def round_bf16(x):
    """float64 -> the nearest bf16, ties to even, as float64."""
    with np.errstate(over="ignore"):
        f = np.asarray(x, np.float64).astype(np.float32)
    u = f.view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)
    return np.where(np.isfinite(f), r, f).astype(np.float64)


def round_to(x, kind):
    with np.errstate(over="ignore"):
        if kind == F16:
            return np.asarray(x).astype(np.float16).astype(np.float64)
        if kind == F32:
            return np.asarray(x).astype(np.float32).astype(np.float64)
    return round_bf16(x)


def quantise(x):
    """(int8 codes, fp32 scales) of the rows along the last axis: a = max|x|, s = fp32(a / 127), r = fp32(127 / a),
    code = rne(fp32(x r)).  In float64 the quotients and products of fp32 values round to fp32 as a direct fp32
    operation would (products are exact, and 53 bits are enough for the quotients)."""
    x = np.asarray(x, np.float32)
    a = np.abs(x).max(-1)
    bad = ~np.isfinite(x).all(-1)
    some = ~bad & (a >= 2.0 ** -100)
    a64 = np.where(some, a, 1).astype(np.float64)
    s = (a64 / 127).astype(np.float32)
    r = (127 / a64).astype(np.float32).astype(np.float64)
    clean = np.where(some[..., None], x, 0).astype(np.float64)
    codes = np.rint((clean * r[..., None]).astype(np.float32)).astype(np.int8)
    return codes, np.where(bad, np.float32(np.nan), np.where(some, s, np.float32(0))).astype(np.float32)


def sequences(offsets, lens, width, page, rows):
    """(first row, rows, length) of each sequence, clamped as the library does."""
    out = []
    for b in range(len(lens)):
        r0 = min(max(int(offsets[b]), 0), rows)
        n = min(max(int(offsets[b + 1]), r0), rows) - r0
        out.append((r0, n, min(max(int(lens[b]), 0), min(width * page, 1 << 30))))
    return out


def slot(table, b, t, page, n_pages):
    """(page id, place) of token t of sequence b, or None for an id out of range."""
    i = int(table[b, t // page])
    return (i, t % page) if 0 <= i < n_pages else None


def write(pool, scales, fmt, table, lens, offsets, x):
    """pool [pages, heads, page, D] as float64 (16-bit formats) or int8; x [rows, heads, D].  Changes pool and scales."""
    n_pages, _, page, _ = pool.shape
    for b, (r0, n, L) in enumerate(sequences(offsets, lens, table.shape[1], page, x.shape[0])):
        for i in range(n):
            t = L - n + i
            at = slot(table, b, t, page, n_pages) if t >= 0 else None
            if at is None:
                continue
            if fmt == KV_I8:
                pool[at[0], :, at[1]], scales[at[0], :, at[1]] = quantise(x[r0 + i])
            else:
                pool[at[0], :, at[1]] = round_to(x[r0 + i], fmt)


def values(pool, scales):
    """What the cache stands for, float64."""
    if scales is None:
        return np.asarray(pool, np.float64)
    return pool.astype(np.float64) * scales.astype(np.float64)[..., None]


def read(pool, scales, table, lens, offsets, rows):
    """[rows, heads, D] float64; rows of no sequence are None's NaN pattern: the mask says which rows are written."""
    n_pages, H, page, D = pool.shape
    out, written = np.zeros((rows, H, D)), np.zeros(rows, bool)
    for b, (r0, n, L) in enumerate(sequences(offsets, lens, table.shape[1], page, rows)):
        for i in range(n):
            t = L - n + i
            written[r0 + i] = True
            if t < 0:
                continue
            at = slot(table, b, t, page, n_pages)
            if at is None:
                out[r0 + i] = np.nan
            else:
                out[r0 + i] = values(pool[at[0], :, at[1]], None if scales is None else scales[at[0], :, at[1]])
    return out, written


def sees(p, t, window, sinks):
    return (t <= p) & ((window == 0) | (t > p - window) | (t < sinks))


def attend(q, kpool, vpool, kscales, vscales, table, lens, offsets, scale, window=0, sinks=0):
    """(out, lse, weight, spread): out [rows, heads, D] and lse [rows, heads] in float64; weight = sum p |v| and
    spread = the largest scale * sum |q| |k| of a row's visible tokens, what an error bound is made of."""
    rows, heads, D = q.shape
    n_pages, H, page, _ = kpool.shape
    G = heads // H
    out, lse = np.zeros((rows, heads, D)), np.full((rows, heads), -np.inf)
    weight, spread = np.zeros((rows, heads, D)), np.zeros((rows, heads))
    for b, (r0, n, L) in enumerate(sequences(offsets, lens, table.shape[1], page, rows)):
        if not n or L <= 0:
            continue
        t = np.arange(L)
        ids = table[b, t // page]
        there = (ids >= 0) & (ids < n_pages)
        k = np.full((L, H, D), np.nan)
        v = np.full((L, H, D), np.nan)
        at = (ids[there], slice(None), (t % page)[there])
        k[there] = values(kpool[at], None if kscales is None else kscales[at])
        v[there] = values(vpool[at], None if vscales is None else vscales[at])
        for i in range(n):
            p = L - n + i
            vis = sees(p, t, window, sinks)
            if not vis.any():
                continue
            kk, vv = k[vis], v[vis]
            for h in range(heads):
                with np.errstate(invalid="ignore", over="ignore"):
                    s = scale * (kk[:, h // G] @ q[r0 + i, h])
                    m = s.max()
                    if m == -np.inf:
                        continue
                    e = np.exp(s - m)
                    z = e.sum()
                    w = e / z
                    # a weight of exactly 0 times an infinity is left to IEEE, as in the definition
                    out[r0 + i, h] = w @ vv[:, h // G]
                    lse[r0 + i, h] = m + np.log(z)
                    weight[r0 + i, h] = w @ np.abs(vv[:, h // G])
                    spread[r0 + i, h] = scale * (np.abs(kk[:, h // G]) @ np.abs(q[r0 + i, h])).max()
    return out, lse, weight, spread
