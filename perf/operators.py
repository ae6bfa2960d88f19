"""The key/value cache and the attention that reads it: cases, plain forms and exact results.

Operators
  store   new keys and values are written into a paged cache (8 bits with one scale per token and head, or 16 bits), then read
          back as the dense rows that the cache now stands for
  read    whole sequences are read back from a paged cache
  attend  rows of queries (one per sequence in decoding, a chunk of a prompt else) attend to the cache, causally, with an
          optional sliding window and a few first tokens that stay visible

`run` computes them in elementary torch operations in 32 bits, or where `own` is true through paper_2606_23419_amd.grinqh.
"""
import math
import random

import torch

own = False

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"i8": 1, "f16": 2, "bf16": 2, "f32": 4}
TINY = 2.0 ** -100  # a row of smaller values is stored as zeros


def case(name, op, B, rows, ctx, ragged=False, hq=32, hk=8, D=128, page=64, fmt="i8", type="f16", window=0, sinks=0, lse=False):
    return {"name": name, "op": op, "B": B, "rows": rows, "ctx": ctx, "ragged": ragged, "hq": hq, "hk": hk, "D": D, "page": page,
            "fmt": fmt, "type": type, "window": window, "sinks": sinks, "lse": lse}


def listed():
    return [
        # one decoded token of one sequence, K and V as the decode VMM leaves them (fp32): latency
        case("store_decode_1", "store", 1, 1, 1023, type="f32"),
        # prompts of unequal odd lengths up to 8191 tokens
        case("store_prompts", "store", 8, 8191, 0, ragged=True, type="bf16", page=32),
        # short sequences of a 16-bit cache of 64-wide heads, gathered into dense rows
        case("read_ragged_16bit", "read", 16, 2047, 0, ragged=True, D=64, page=16, fmt="f16", type="f16"),
        # one long 8-bit context as dense fp16
        case("read_long", "read", 1, 131072, 0),
        # a decoded token after a short prompt: latency
        case("decode_77", "attend", 1, 1, 76),
        # a decoded token at the far end of a long context: few rows, the length has to be split
        case("decode_long", "attend", 1, 1, 131071),
        # a batch of sequences of unequal lengths
        case("decode_batch", "attend", 32, 1, 8190, ragged=True, page=16, type="bf16"),
        # decoding with a window and sinks over a 16-bit cache, pages behind the window given back
        case("decode_window", "attend", 16, 1, 32767, fmt="f16", window=4096, sinks=4),
        # a prompt of 2048 tokens from its start, 16-bit cache
        case("prompt_2048", "attend", 1, 2048, 0, fmt="f16"),
        # chunks of unequal odd lengths, seven query heads to a key head, statistics returned too
        case("chunk_ragged", "attend", 6, 777, 5001, ragged=True, hq=28, hk=4, page=16, lse=True),
        # a chunk of a long prompt under a window with sinks, bf16
        case("chunk_window", "attend", 1, 4096, 12288, fmt="bf16", type="bf16", page=128, window=2048, sinks=4),
        # a large chunk over a long 8-bit context
        case("chunk_long", "attend", 1, 4096, 32768),
    ]


LARGEST = 32 * 4096 * 36864  # query heads x rows x keys of the largest plain pass
TOKENS = 131072              # tokens of the largest cache pass, at 8 heads of 128


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    c = case("", rng.choice(["store", "read", "attend", "attend", "attend"]), 1, 1, 0)
    del c["name"]
    c["hq"], c["hk"] = rng.choice([(32, 8), (32, 8), (16, 4), (8, 1), (12, 12), (28, 4), (40, 8)])
    c["D"], c["page"] = rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 128, 256])
    c["fmt"] = rng.choice(["i8", "i8", "f16", "bf16"])
    c["B"], c["ragged"] = log(1, 64), rng.random() < 0.6
    most = TOKENS * 8 * 128 // (c["hk"] * c["D"])  # tokens in all
    if c["op"] != "attend":
        c["type"] = rng.choice(["f16", "bf16", "f32"])
        c["rows"] = log(1, max(2, min(16384, most // 2 // c["B"])))
        c["ctx"] = log(1, 4096) - 1 if c["op"] == "store" else 0
        return c
    c["type"] = rng.choice(["f16", "bf16"]) if c["fmt"] == "i8" else c["fmt"]
    c["rows"] = 1 if rng.random() < 0.4 else log(1, 4096)
    c["ctx"] = log(1, 65536) - 1
    while c["B"] * c["hq"] * c["rows"] * (c["rows"] + c["ctx"]) > LARGEST // 4 or c["B"] * (c["rows"] + c["ctx"]) > most:
        k = max(["B", "rows", "ctx"], key=lambda k: c[k])
        c[k] = max(1, c[k] * 2 // 3)
    if rng.random() < 0.35:
        c["window"], c["sinks"] = log(16, 8192), rng.choice([0, 1, 4, 64])
    c["lse"] = rng.random() < 0.3
    return c


def lengths(c):
    """(rows, total length) of each sequence: a matter of the case alone. The first has the case's own."""
    r = random.Random("%(B)d %(rows)d %(ctx)d %(hq)d %(D)d" % c)
    part = [1.0] + [r.random() ** 2 if c["ragged"] else 1.0 for _ in range(c["B"] - 1)]
    rows = [c["rows"] if c["rows"] == 1 else int(c["rows"] * p) for p in part]
    return [(n, n + (int(c["ctx"] * r.random()) if c["ragged"] and i else c["ctx"])) for i, n in enumerate(rows)]


def visible(n, L, W, S):
    """Pairs of row and visible token, and tokens that any row sees, of n rows at the end of L tokens."""
    first = L - n
    if not W or not n:
        return n * first + n * (n + 1) // 2, L if n else 0
    ramp = max(0, min(n, W - first))  # rows that see all before them
    pairs = ramp * first + ramp * (ramp + 1) // 2 + (n - ramp) * W
    lo = max(0, first - W + 1)  # the first row's window starts here
    pairs += sum(min(S, max(0, p - W + 1)) for p in range(first + ramp, L)) if S else 0
    return pairs, L - lo + min(S, lo)


def work(c):
    total, T = lengths(c), sum(n for n, _ in lengths(c))
    held = c["D"] * BYTES[c["fmt"]] + (4 if c["fmt"] == "i8" else 0)  # one head of one token in the cache
    dense = c["D"] * BYTES[c["type"]]
    if c["op"] == "store":  # rows in, cache out, and the rows that are returned
        return {"bytes": 2 * T * c["hk"] * (2 * dense + held), "flops": 0}
    if c["op"] == "read":
        return {"bytes": 2 * T * c["hk"] * (dense + held), "flops": 0}
    seen = [visible(n, L, c["window"], c["sinks"]) for n, L in total]
    return {"bytes": 2 * c["hk"] * held * sum(s for _, s in seen) + T * c["hq"] * (2 * dense + 4 * c["lse"]),
            "flops": 4 * c["D"] * c["hq"] * sum(p for p, _ in seen)}


def normal(shape, gen, spread=None):
    x = torch.randn(shape, generator=gen, device="cuda")
    return x if spread is None else x.mul_(spread)


def quantise(x):
    """(codes, scales) of the rows along the last axis of fp32 x."""
    a = x.abs().amax(-1, keepdim=True)
    some = a >= TINY
    a = torch.where(some, a, torch.ones_like(a))
    r = torch.where(some, torch.full_like(a, 127.0) / a, torch.zeros_like(a))
    s = torch.where(some, a / torch.full_like(a, 127.0), torch.zeros_like(a))
    return (x * r).round().to(torch.int8), s.squeeze(-1)


def prepare(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    seqs = lengths(c)
    P, H, D = c["page"], c["hk"], c["D"]
    width = max(1, max(-(-L // P) for _, L in seqs))  # pages of the longest sequence
    n_pages = sum(-(-L // P) for _, L in seqs) + 3
    # the sequences' pages in no order, as a server's free list hands them out
    perm = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((c["B"], width), -1, dtype=torch.int32)
    at = 0
    for b, (n, L) in enumerate(seqs):
        k = -(-L // P)
        table[b, :k] = torch.arange(at, at + k, dtype=torch.int32)
        at += k
    held = table >= 0
    if c["window"]:  # pages that no row sees any more have been given back
        for b, (n, L) in enumerate(seqs):
            lo = max(0, L - n - c["window"] + 1) // P
            held[b, min(lo, -(-c["sinks"] // P)):lo] = False
    table, held = table.cuda(), held.cuda()
    table = torch.where(held, perm[table.clamp(min=0).long()], torch.full_like(table, -1))
    offsets = [0]
    for n, _ in seqs:
        offsets.append(offsets[-1] + n)
    st = {"c": c, "table": table, "lens": torch.tensor([L for _, L in seqs], dtype=torch.int32, device="cuda"),
          "offsets": torch.tensor(offsets, dtype=torch.int32, device="cuda"), "T": offsets[-1],
          "max_rows": max(n for n, _ in seqs), "max_len": max(L for _, L in seqs)}
    # keys have a few channels of larger values, as trained models' keys do
    spread = torch.ones(D, device="cuda")
    spread[::29] = 4.0
    for name in ("k", "v"):
        wide = spread if name == "k" else None
        if c["op"] == "store":
            st["new_" + name] = normal((st["T"], H, D), gen, wide).to(TYPES[c["type"]])
            pool = torch.zeros((n_pages, H, P, D), device="cuda", dtype=torch.int8 if c["fmt"] == "i8" else TYPES[c["fmt"]])
            scale = torch.zeros((n_pages, H, P), device="cuda") if c["fmt"] == "i8" else None
        elif c["fmt"] == "i8":
            pool, scale = quantise(normal((n_pages, H, P, D), gen, wide))
        else:
            pool, scale = normal((n_pages, H, P, D), gen, wide).to(TYPES[c["fmt"]]), None
        st[name], st[name + "_scale"] = pool, scale
    if c["op"] == "attend":
        st["q"] = normal((st["T"], c["hq"], D), gen).to(TYPES[c["type"]])
        if c["lse"]:
            st["lse"] = torch.empty((st["T"], c["hq"]), device="cuda")
    return st


def handles(st):
    """What a program makes once for its cache and its batch: descriptors, output buffers and the workspace."""
    from paper_2606_23419_amd import grinqh as g

    c = st["c"]
    desc = g.make_kv_desc({"i8": g.GRINQH_KV_I8, "f16": g.GRINQH_KV_F16, "bf16": g.GRINQH_KV_BF16}[c["fmt"]],
                          c["hk"], c["D"], c["page"], st["k"].shape[0])
    what = (desc, g.KvCache(st["k"], st["v"], st["k_scale"], st["v_scale"]), g.KvBatch(st["table"], st["lens"], st["offsets"]))
    if c["op"] == "attend":
        size = g.grinqh_attend_workspace_bytes(desc, c["hq"], c["B"], st["T"], max_rows=st["max_rows"], max_len=st["max_len"],
                                               window=c["window"], sinks=c["sinks"])
        kept = {"out": torch.empty_like(st["q"]), "workspace": torch.empty(size, dtype=torch.uint8, device="cuda")}
    else:
        kept = {x: torch.empty((st["T"], c["hk"], c["D"]), dtype=TYPES[c["type"]], device="cuda") for x in ("k", "v")}
    return g, what, kept


def run_own(st):
    if "handles" not in st:
        st["handles"] = handles(st)
    g, what, kept = st["handles"]
    c = st["c"]
    if c["op"] == "attend":
        out = g.grinqh_attend(*what, st["q"], window=c["window"], sinks=c["sinks"], max_rows=st["max_rows"],
                              max_len=st["max_len"], lse=st.get("lse"), **kept)
        return {"out": out, "lse": st.get("lse")}
    if c["op"] == "store":
        g.grinqh_kv_write(*what, st["new_k"], st["new_v"])
    k, v = g.grinqh_kv_read(*what, st["T"], dtype=TYPES[c["type"]], **kept)
    return {"k": k, "v": v, "scales": [st["k_scale"], st["v_scale"]] if c["op"] == "store" else None}


def slots(st):
    """(page, place in the page) of each row."""
    row = torch.arange(st["T"], device="cuda")
    b = torch.searchsorted(st["offsets"], row, right=True) - 1
    pos = st["lens"][b] - st["offsets"][b + 1] + row
    return st["table"][b, pos // st["c"]["page"]].long(), pos % st["c"]["page"]


def run_cache(st):
    """store and read, in plain torch."""
    c = st["c"]
    page, place = slots(st)
    got = {"scales": [st["k_scale"], st["v_scale"]] if c["op"] == "store" else None}

    def one(name):
        pool, scale = st[name], st[name + "_scale"]
        if c["op"] == "store":
            x = st["new_" + name].float()
            if scale is not None:
                x, s = quantise(x)
                scale[page, :, place] = s
            pool[page, :, place] = x.to(pool.dtype)
        x = pool[page, :, place].float()
        return (x if scale is None else x * scale[page, :, place].unsqueeze(-1)).to(TYPES[c["type"]])

    return got | {"k": one("k"), "v": one("v")}


def run_attend(st):
    """attend, in plain torch: every sequence padded to the longest."""
    c = st["c"]
    B, H, D, G, n, L = c["B"], c["hk"], c["D"], c["hq"] // c["hk"], st["max_rows"], st["max_len"]
    t = torch.arange(L, device="cuda")
    page = st["table"][:, t // c["page"]].clamp(min=0).long()  # [B, L]

    def dense(name):
        x = st[name][page, :, t % c["page"]].float()  # [B, L, H, D]
        if st[name + "_scale"] is not None:
            x = x * st[name + "_scale"][page, :, t % c["page"]].unsqueeze(-1)
        return x.permute(0, 2, 1, 3).contiguous()

    i = torch.arange(n, device="cuda")
    count = st["offsets"][1:] - st["offsets"][:-1]
    there = i < count[:, None]  # [B, n]
    rows = (st["offsets"][:-1, None] + i).clamp(max=max(0, st["T"] - 1))
    q = st["q"][rows].float().reshape(B, n, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, n * G, D)
    pos = st["lens"][:, None] - count[:, None] + i
    sees = (t <= pos[..., None]) & there[..., None]  # [B, n, L]
    if c["window"]:
        sees &= (t > pos[..., None] - c["window"]) | (t < c["sinks"])
    s = torch.matmul(q, dense("k").transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(D)).view(B, H, n, G, L)
    s.masked_fill_(~sees[:, None, :, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    s.sub_(m).exp_()
    l = s.sum(-1, keepdim=True)
    o = torch.matmul(s.view(B, H, n * G, L), dense("v")).view(B, H, n, G, D) / torch.where(l > 0, l, torch.ones_like(l))
    out = o.permute(0, 2, 1, 3, 4).reshape(B, n, c["hq"], D)[there].to(st["q"].dtype)
    if not c["lse"]:
        return {"out": out, "lse": None}
    return {"out": out, "lse": (m + l.log()).squeeze(-1).permute(0, 2, 1, 3).reshape(B, n, c["hq"])[there]}


def run(st):
    if own:
        return run_own(st)
    return run_attend(st) if st["c"]["op"] == "attend" else run_cache(st)


def exact(c, seed):
    """The same from the definitions, in 64 bits, one sequence and one head at a time."""
    st = prepare(c, seed)
    P, H, D, G = c["page"], c["hk"], c["D"], c["hq"] // c["hk"]
    seqs, first = lengths(c), 0
    table = st["table"].cpu()
    if c["op"] == "store":
        got = {"scales": None}
        for name in ("k", "v"):
            x = st["new_" + name].double()
            if c["fmt"] == "i8":
                s = x.abs().amax(-1, keepdim=True) / 127
                x = torch.where(s > 0, torch.round(x / s), torch.zeros_like(x)) * s
            elif c["fmt"] != c["type"]:
                x = x.to(TYPES[c["fmt"]]).double()  # the cache's type rounds
            got[name] = x
        return got
    pages = {}
    for name in ("k", "v"):
        x = st[name].double()
        pages[name] = x if c["fmt"] != "i8" else x * st[name + "_scale"].double()[..., None]
    got = {"k": [], "v": []} if c["op"] == "read" else {"out": [], "lse": []}
    for b, (n, L) in enumerate(seqs):
        ids = table[b, :-(-L // P)].clamp(min=0).long().cuda()
        whole = {name: x[ids].permute(0, 2, 1, 3).reshape(-1, H, D)[:L] for name, x in pages.items()}
        if c["op"] == "read":
            got["k"].append(whole["k"][L - n:])
            got["v"].append(whole["v"][L - n:])
            continue
        q = st["q"][first:first + n].double()
        first += n
        out, lse = torch.zeros((n, c["hq"], D), dtype=torch.float64, device="cuda"), torch.zeros((n, c["hq"]), dtype=torch.float64, device="cuda")
        p, t = torch.arange(L - n, L, device="cuda")[:, None], torch.arange(L, device="cuda")[None]
        hidden = t > p
        if c["window"]:
            hidden |= (t <= p - c["window"]) & (t >= c["sinks"])
        for h in range(c["hq"]):
            s = (q[:, h] @ whole["k"][:, h // G].T) / math.sqrt(D)
            s[hidden] = -math.inf
            if n:
                lse[:, h] = torch.logsumexp(s, -1)
                out[:, h] = torch.exp(s - lse[:, h, None]) @ whole["v"][:, h // G].contiguous()
        got["out"].append(out)
        got["lse"].append(lse)
    got = {name: torch.cat(x) for name, x in got.items()}
    if c["op"] == "read":
        return got | {"scales": None}
    return {"out": got["out"], "lse": got["lse"] if c["lse"] else None}
