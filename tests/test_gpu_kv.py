"""The key/value cache and the attention over it against the float64 oracle, through the binding.

Error bounds.  kv_write and kv_read are compared bit for bit.  For attend, per element,
  |out - ref| <= u_out |ref| + (u_p + 2 d + 2^-14) sum_t p_t |v_t| + 2^-23 max |v|
with u_out and u_p the half-ulp of the output's type and of the weights' type (2^-11 in fp16, which has 11 significant bits,
2^-8 in bf16, which has 8: the weight of each token is rounded once, and the sum that divides is of the unrounded ones), d = 2 D 2^-24 scale sum |q||k| the
fp32 error of a score (an absolute error d of a score is a relative error d of its weight, and as much of the sum), 2^-14 for
exp and the scores' products by constants at scores up to a few hundred, and the last term for weights under fp16's
normal range.  lse: d + 2^-20 (1 + |ref|)."""
import numpy as np
import pytest

from oracle import kv_oracle as kv

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def g():
    from paper_2606_23419_amd import grinqh
    return grinqh


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available()
    return t


def dtype(torch, kind):
    return {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32, "i8": torch.int8}[kind]


def up(torch, x, kind):
    """A float64 array whose values `kind` holds exactly, on the device."""
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float64)).to(dtype(torch, kind)).cuda()


def down(t):
    return t.detach().cpu().double().numpy()


class Case:
    """Sequences of (rows, length) over a paged cache of random values; pages in random order."""

    def __init__(self, g, torch, seqs, fmt="i8", H=2, G=4, D=128, page=16, type="f16", seed=0, spread=1.0, spare=2,
                 fill=None):
        self.g, self.torch, self.fmt, self.type, self.H, self.D, self.page = g, torch, fmt, type, H, D, page
        rng = self.rng = np.random.default_rng(seed)
        self.rows, self.heads, self.B = sum(n for n, _ in seqs), H * G, len(seqs)
        need = [-(-L // page) for _, L in seqs]
        self.width, self.n_pages = max(1, max(need)), sum(need) + spare
        ids = rng.permutation(self.n_pages)
        self.table = rng.integers(-9, 3 * self.n_pages, (self.B, self.width)).astype(np.int32)  # what no one may follow
        at = 0
        for b, k in enumerate(need):
            self.table[b, :k] = ids[at:at + k]
            at += k
        self.lens = np.array([L for _, L in seqs], np.int32)
        self.offsets = np.cumsum([0] + [n for n, _ in seqs]).astype(np.int32)
        self.pool, self.scales = {}, {"k": None, "v": None}
        for name in "kv":
            x = rng.standard_normal((self.n_pages, H, page, D)) * spread
            if fmt == "i8":
                self.pool[name], self.scales[name] = kv.quantise(x)
            else:
                self.pool[name] = kv.round_to(x, fmt)
        if fill is not None:  # every place that holds no token of any sequence
            used = np.zeros((self.n_pages, page), bool)
            for b, (n, L) in enumerate(seqs):
                for t in range(L):
                    used[self.table[b, t // page], t % page] = True
            for name in "kv":
                if fmt == "i8":
                    self.pool[name] = np.where(used[:, None, :, None], self.pool[name], np.int8(-128))
                    self.scales[name] = np.where(used[:, None], self.scales[name], np.float32(fill))
                else:
                    self.pool[name] = np.where(used[:, None, :, None], self.pool[name], fill)
        self.q = kv.round_to(rng.standard_normal((self.rows, self.heads, D)), type)

    def upload(self):
        g, torch = self.g, self.torch
        self.desc = g.make_kv_desc({"i8": g.GRINQH_KV_I8, "f16": g.GRINQH_KV_F16, "bf16": g.GRINQH_KV_BF16}[self.fmt],
                                   self.H, self.D, self.page, self.n_pages)
        s = [torch.from_numpy(self.scales[n]).cuda() if self.fmt == "i8" else None for n in "kv"]
        self.cache = g.KvCache(up(torch, self.pool["k"], self.fmt), up(torch, self.pool["v"], self.fmt), *s)
        self.batch = g.KvBatch(torch.from_numpy(self.table).cuda(), torch.from_numpy(self.lens).cuda(),
                               torch.from_numpy(self.offsets).cuda())
        return self

    def attend(self, q=None, lse=True, **kw):
        torch = self.torch
        q = up(torch, self.q, self.type) if q is None else q
        out = torch.full((self.rows, self.heads, self.D), 777.0, dtype=q.dtype, device="cuda")
        z = torch.full((self.rows, self.heads), 777.0, device="cuda") if lse else None
        self.g.grinqh_attend(self.desc, self.cache, self.batch, q, out=out, lse=z, **kw)
        return out, z

    def want(self, window=0, sinks=0, scale=None):
        return kv.attend(self.q, self.pool["k"], self.pool["v"], self.scales["k"], self.scales["v"], self.table, self.lens,
                         self.offsets, self.D ** -0.5 if scale is None else scale, window, sinks)

    def check(self, out, lse, window=0, sinks=0, scale=None):
        ref, ref_lse, weight, spread = self.want(window, sinks, scale)
        u = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}
        d = 2 * self.D * 2.0 ** -24 * spread[..., None]
        bound = u[self.type] * np.abs(ref) + (u["bf16" if self.fmt == "bf16" else "f16"] + 2 * d + 2.0 ** -14) * weight
        vals = np.abs(kv.values(self.pool["v"], self.scales["v"]))
        bound += 2.0 ** -23 * np.max(vals, initial=0, where=np.isfinite(vals))
        got = down(out)
        assert np.array_equal(np.isnan(got), np.isnan(ref))
        with np.errstate(invalid="ignore"):
            far = np.where(np.isfinite(ref), np.abs(got - ref) - bound, np.where(np.isnan(ref) | (got == ref), -1, np.inf))
        assert far.max(initial=-1) <= 0, (far.max(), np.unravel_index(far.argmax(), far.shape))
        if lse is not None:
            got = down(lse)
            assert np.array_equal(np.isnan(got), np.isnan(ref_lse)) and np.array_equal(got == -np.inf, ref_lse == -np.inf)
            fine = np.isfinite(ref_lse)
            assert (np.abs(got - ref_lse)[fine] <= (d[..., 0] + 2.0 ** -20 * (1 + np.abs(ref_lse)))[fine]).all()


FORMATS = [("i8", "f16"), ("i8", "bf16"), ("f16", "f16"), ("bf16", "bf16")]

# ------------------------------------------------------------------ cache --
SEQS = [(5, 5), (0, 7), (1, 40), (33, 100), (9, 4), (2, 2), (64, 64)]   # the fifth has rows before its first token


def rows_of(torch, rng, rows, H, D, type, layout, scale=1.0):
    """Random rows as float64 and on the device, as a view of one of several layouts."""
    x = kv.round_to(rng.standard_normal((rows, H, D)) * scale, type)
    t = up(torch, x, type)
    if layout == "fused":      # a slice of wider rows
        wide = torch.full((rows, H * D + 64), 9.0, dtype=t.dtype, device="cuda")
        wide[:, 32:32 + H * D] = t.view(rows, H * D)
        t = wide[:, 32:32 + H * D].view(rows, H, D)
    elif layout == "heads":    # heads first
        t = t.permute(1, 0, 2).contiguous().permute(1, 0, 2)
    return x, t


@pytest.mark.parametrize("fmt", ["i8", "f16", "bf16"])
@pytest.mark.parametrize("type", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("D,H,page,layout", [(128, 8, 16, "plain"), (64, 3, 1, "fused"), (128, 1, 64, "heads"), (64, 5, 8, "plain")])
def test_write_and_read(g, torch, fmt, type, D, H, page, layout):
    c = Case(g, torch, SEQS, fmt=fmt, H=H, D=D, page=page, type=type if type != "f32" else "f16", seed=3)
    c.table[3, 3 // page] = -1          # not where any row goes
    if page <= 16:
        c.table[6, 20 // page] = c.n_pages   # rows of the last sequence that have no page
    c.upload()
    rng = np.random.default_rng(4)
    x = {n: rows_of(torch, rng, c.rows, H, D, type, layout, 3.0) for n in "kv"}
    g.grinqh_kv_write(c.desc, c.cache, c.batch, x["k"][1], x["v"][1])
    for n in "kv":
        pool, scales = c.pool[n].copy(), None if c.scales[n] is None else c.scales[n].copy()
        kv.write(pool, scales, fmt, c.table, c.lens, c.offsets, x[n][0])
        assert np.array_equal(down(getattr(c.cache, n)), pool.astype(np.float64))
        if fmt == "i8":
            assert np.array_equal(down(getattr(c.cache, n + "_scale")), scales.astype(np.float64))
        c.pool[n], c.scales[n] = pool, scales
    for out in ("f16", "bf16", "f32"):
        got = g.grinqh_kv_read(c.desc, c.cache, c.batch, c.rows, dtype=dtype(torch, out))
        for n, t in zip("kv", got):
            ref, written = kv.read(c.pool[n], c.scales[n], c.table, c.lens, c.offsets, c.rows)
            assert written.all()
            if fmt == "i8":   # the product of code and scale is one fp32 operation
                ref = ref.astype(np.float32).astype(np.float64)
            assert np.array_equal(down(t), kv.round_to(ref, out), equal_nan=True)


def test_write_extreme_rows(g, torch):
    c = Case(g, torch, [(8, 8)], H=1, D=64, page=4).upload()
    x = np.zeros((8, 1, 64), np.float32)
    x[0, 0, 3], x[1, 0, 5], x[2, 0, 7], x[3, 0, 63], x[4, 0, 0] = np.nan, np.inf, 2.0 ** -101, 2.0 ** -100, -3e38
    x[5, 0, :2] = 1e-30, -1e-30
    x[6] = np.nan
    x[7, 0, 1] = -np.inf
    t = torch.from_numpy(x).cuda()
    g.grinqh_kv_write(c.desc, c.cache, c.batch, t, t)
    kv.write(c.pool["k"], c.scales["k"], "i8", c.table, c.lens, c.offsets, x)
    assert np.array_equal(down(c.cache.k), c.pool["k"].astype(np.float64))
    assert np.array_equal(down(c.cache.k_scale), c.scales["k"].astype(np.float64), equal_nan=True)
    assert np.isnan(c.scales["k"]).sum() == 4


def test_write_casts_to_16_bits_as_torch_does(g, torch):
    x = torch.tensor([0.0, -0.0, 1e-8, 6e-8, 65519.0, 65520.0, 3.4e38, -3.4e38, float("inf"), -float("inf"), float("nan"), 1e-45,
                      1 + 2.0 ** -11, 1 + 3 * 2.0 ** -11, 1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8]).repeat(4).view(1, 1, 64).cuda()
    for fmt in ("f16", "bf16"):
        c = Case(g, torch, [(1, 1)], fmt=fmt, H=1, D=64, page=4, type=fmt).upload()
        g.grinqh_kv_write(c.desc, c.cache, c.batch, x, x)
        got = c.cache.k[c.table[0, 0], 0, 0].cpu()
        want = x.to(dtype(torch, fmt)).cpu().view(64)
        assert torch.equal(torch.nan_to_num(got, nan=5.0), torch.nan_to_num(want, nan=5.0))
        assert torch.equal(torch.isnan(got), torch.isnan(want))


def test_rows_of_no_sequence_are_left_alone(g, torch):
    c = Case(g, torch, [(3, 6), (2, 9)], H=2, D=64, page=4)
    c.rows += 4
    c.q = np.concatenate([c.q, c.q[:4]])
    c.offsets = c.offsets + 2           # two rows before the first sequence and two behind the last
    c.upload()
    k = torch.full((9, 2, 64), 5.0, dtype=torch.float16, device="cuda")
    v = k.clone()
    g.grinqh_kv_read(c.desc, c.cache, c.batch, 9, k=k, v=v)
    out, lse = c.attend()
    ref, written = kv.read(c.pool["k"], c.scales["k"], c.table, c.lens, c.offsets, 9)
    assert written.tolist() == [False] * 2 + [True] * 5 + [False] * 2
    assert (down(k)[~written] == 5).all() and (down(out)[~written] == 777).all() and (down(lse)[~written] == 777).all()
    assert np.abs(down(k)[written] - ref[written]).max() < 0.01
    before = c.cache.k.clone()
    g.grinqh_kv_write(c.desc, c.cache, c.batch, k, v)
    changed = (down(c.cache.k) != down(before)).any(-1).any(1).sum()
    assert changed <= 5


def test_offsets_and_lengths_out_of_range_are_clamped(g, torch):
    for offsets, lens in [([-5, 3, 100], [6, 9]), ([0, 4, 2], [6, 9]), ([0, 2, 4], [1000, -3]), ([9, 9, 9], [6, 9]),
                          ([0, 2, 4], [2 ** 31 - 1, 9])]:
        c = Case(g, torch, [(2, 8), (2, 12)], H=2, D=64, page=4)
        c.offsets, c.lens = np.array(offsets, np.int32), np.array(lens, np.int32)
        c.table[0, 2:] = -1
        c.upload()
        out, lse = c.attend(max_rows=4, max_len=12)
        written = np.zeros(c.rows, bool)
        for r0, n, _ in kv.sequences(c.offsets, c.lens, c.width, c.page, c.rows):
            written[r0:r0 + n] = True
        ref, ref_lse, _, _ = c.want()
        got = down(out)
        assert (got[~written] == 777).all()
        # rows that two clamped sequences share may hold either's result; none is shared here
        assert np.array_equal(np.isnan(got[written]), np.isnan(ref[written]))
        assert np.nanmax(np.abs(got - ref)[written], initial=0) < 0.01


def test_slots_past_32_bits(g, torch):
    """A cache of over 2^31 values and 2^32 bytes of K: the last pages are written, read and attended to."""
    page, H, D = 256, 8, 128
    n_pages = (1 << 31) // (page * H * D) + 40
    desc = g.make_kv_desc(g.GRINQH_KV_F16, H, D, page, n_pages)
    cache = g.KvCache(*[torch.empty((n_pages, H, page, D), dtype=torch.float16, device="cuda") for _ in "kv"], None, None)
    table = torch.tensor([[n_pages - 1, 3, n_pages - 2]], dtype=torch.int32, device="cuda")
    L = 600
    batch = g.KvBatch(table, torch.tensor([L], dtype=torch.int32, device="cuda"), torch.tensor([0, L], dtype=torch.int32, device="cuda"))
    k, v = [torch.randn((L, H, D), device="cuda").to(torch.float16) for _ in "kv"]
    g.grinqh_kv_write(desc, cache, batch, k, v)
    assert torch.equal(cache.k[n_pages - 1, :, 255], k[255]) and torch.equal(cache.v[n_pages - 2, :, 87], v[599])
    rk, rv = g.grinqh_kv_read(desc, cache, batch, L)
    assert torch.equal(rk, k) and torch.equal(rv, v)
    q = torch.randn((L, H, D), device="cuda").to(torch.float16)
    out = g.grinqh_attend(desc, cache, batch, q)
    one = g.KvBatch(table, batch.seq_lens, torch.tensor([0, 1], dtype=torch.int32, device="cuda"))
    last = g.grinqh_attend(desc, cache, one, q[-1:])
    s = torch.einsum("hd,lhd->hl", q[-1].cpu().double(), k.cpu().double()) * D ** -0.5
    want = torch.einsum("hl,lhd->hd", s.softmax(-1), v.cpu().double())
    for got in (out[-1], last[0]):
        assert (got.cpu().double() - want).abs().max() < 2e-3


# -------------------------------------------------------------- attention --
@pytest.mark.parametrize("fmt,type", FORMATS)
@pytest.mark.parametrize("D,H,G,page", [(128, 2, 4, 16), (64, 3, 1, 64), (128, 1, 7, 1), (64, 2, 5, 128)])
@pytest.mark.parametrize("seqs", [
    [(1, 1)],
    [(1, 77), (1, 0), (1, 32), (1, 33), (1, 200)],          # one row each; a sequence of nothing
    [(5, 5), (0, 7), (3, 40), (33, 100), (9, 4), (64, 64)],  # chunks, no rows, rows before the first token
    [(130, 131), (1, 300), (257, 400)],
])
def test_attend(g, torch, fmt, type, D, H, G, page, seqs):
    c = Case(g, torch, seqs, fmt=fmt, type=type, D=D, H=H, G=G, page=page, seed=len(seqs), fill=float("nan")).upload()
    c.check(*c.attend())


@pytest.fixture(params=["rows", "tile", "tilex3", "rowsx3"])
def forced(g, request):
    """Every kernel on its own, and sequences split in three whatever their size."""
    kernel = {"rows": g.GRINQH_ATTEND_ROWS, "tile": g.GRINQH_ATTEND_TILE}
    name, _, splits = request.param.partition("x")
    g.grinqh_set_option(g.GRINQH_OPT_ATTEND_KERNEL, kernel[name])
    g.grinqh_set_option(g.GRINQH_OPT_ATTEND_SPLITS, int(splits or 0))
    yield request.param
    g.grinqh_set_option(g.GRINQH_OPT_ATTEND_KERNEL, 0)
    g.grinqh_set_option(g.GRINQH_OPT_ATTEND_SPLITS, 0)


@pytest.mark.parametrize("fmt,type", FORMATS)
@pytest.mark.parametrize("D,G,page", [(128, 4, 16), (64, 3, 2)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 5)])
def test_every_kernel(g, torch, forced, fmt, type, D, G, page, window, sinks):
    seqs = [(1, 1), (90, 300), (0, 3), (1, 500), (9, 4), (64, 64)]
    c = Case(g, torch, seqs, fmt=fmt, type=type, D=D, H=2, G=G, page=page, fill=float("nan")).upload()
    out, lse = c.attend(window=window, sinks=sinks, max_rows=90, max_len=500)
    c.check(out, lse, window, sinks)


@pytest.mark.parametrize("fmt,type", [("f16", "f16"), ("bf16", "bf16"), ("i8", "f16")])
def test_masked_infinities_in_every_kernel(g, torch, forced, fmt, type):
    """Values of all three kinds at one channel each, seen by the later rows of a chunk only."""
    n, L, window = 100, 130, 40
    bad = {3: float("inf"), 40: -float("inf"), 77: float("nan")}
    for t in (35, 64, 99, 127):
        c = Case(g, torch, [(n, L)], fmt=fmt, type=type, H=1, G=2, page=16, seed=5)
        if fmt == "i8":
            c.scales["v"][c.table[0, t // 16], :, t % 16] = float("nan")
        else:
            for d, x in bad.items():
                c.pool["v"][c.table[0, t // 16], :, t % 16, d] = x
        c.upload()
        got = down(c.attend(window=window)[0])
        seen = kv.sees(np.arange(L - n, L), t, window, 0)
        assert np.isfinite(got[~seen]).all()
        if fmt == "i8":
            assert np.isnan(got[seen]).all()
        else:
            for d, x in bad.items():
                assert np.array_equal(got[seen][..., d], np.full_like(got[seen][..., d], x), equal_nan=True)
            assert np.isfinite(np.delete(got, list(bad), axis=-1)).all()


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 0), (16, 4), (63, 1), (64, 64), (100, 7), (65, 200), (1000, 4)])
@pytest.mark.parametrize("fmt,type", [("i8", "f16"), ("bf16", "bf16")])
def test_window_and_sinks(g, torch, fmt, type, window, sinks):
    c = Case(g, torch, [(1, 300), (40, 333), (3, 17), (150, 150), (2, 1)], fmt=fmt, type=type, page=8, fill=float("inf"))
    # pages that no row sees have been given back
    for b, (n, L) in enumerate([(1, 300), (40, 333), (3, 17), (150, 150), (2, 1)]):
        lo = max(0, L - n - window + 1) // 8
        c.table[b, min(lo, -(-sinks // 8)):lo] = [-1, 1 << 30][b & 1]
    c.upload()
    c.check(*c.attend(window=window, sinks=sinks), window, sinks)


@pytest.mark.parametrize("seqs,H,G", [([(1, 9000)], 1, 4), ([(1, 5003), (1, 64), (1, 12000)], 2, 8), ([(3, 7001)], 2, 1), ([(1, 3001)], 1, 40),
                                      ([(70, 6000)], 1, 2)])
@pytest.mark.parametrize("fmt,type", [("i8", "bf16"), ("f16", "f16")])
def test_long_context(g, torch, fmt, type, seqs, H, G):
    c = Case(g, torch, seqs, fmt=fmt, type=type, H=H, G=G, page=32).upload()
    out, lse = c.attend(max_rows=max(n for n, _ in seqs), max_len=max(L for _, L in seqs))
    c.check(out, lse)
    # without lse, the same bits
    assert self_equal(torch, c.attend(lse=False, max_rows=max(n for n, _ in seqs), max_len=max(L for _, L in seqs))[0], out)


def self_equal(torch, a, b):
    return torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("hints", [(1, 1), (1, 1 << 30), (1 << 24, 1), (3, 100), (1 << 24, 1 << 30)])
def test_estimates_shape_the_launch_only(g, torch, hints):
    c = Case(g, torch, [(1, 700), (90, 900), (300, 310)], page=16).upload()
    c.check(*c.attend(max_rows=hints[0], max_len=hints[1]))


@pytest.mark.parametrize("fmt,type", FORMATS)
@pytest.mark.parametrize("n,L", [(1, 130), (4, 130), (150, 200)])
def test_bad_page_ids_poison_only_the_rows_that_see_them(g, torch, fmt, type, n, L):
    c = Case(g, torch, [(n, L), (n, L)], fmt=fmt, type=type, page=16)
    c.table[0, 64 // 16], c.table[1, (L - 1) // 16] = -1, c.n_pages
    c.upload()
    out, lse = c.attend()
    c.check(out, lse)
    nan = np.isnan(down(out)).any((1, 2))
    assert nan[:n].any() and nan[n:].any()
    assert n < 100 or (not nan[:n].all() and not nan[n:].all())
    # behind a window they are not seen
    out, lse = c.attend(window=17, sinks=3)
    c.check(out, lse, 17, 3)


@pytest.mark.parametrize("fmt,type", FORMATS)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("n,L", [(3, 70), (40, 70), (150, 150)])
@pytest.mark.parametrize("window", [0, 20])
def test_later_and_windowed_out_tokens_never_reach_a_row(g, torch, fmt, type, bad, n, L, window):
    clean = Case(g, torch, [(n, L)], fmt=fmt, type=type, H=1, G=2, page=16, seed=5).upload()
    base, base_lse = clean.attend(window=window)
    clean.check(base, base_lse, window)
    for name in "kv":
        for t in (L - 1, L - 2 if n > 2 else L - 1, max(0, L - n - 1)):
            c = Case(g, torch, [(n, L)], fmt=fmt, type=type, H=1, G=2, page=16, seed=5)
            if fmt == "i8":
                c.scales[name][c.table[0, t // 16], :, t % 16] = bad
            else:
                c.pool[name][c.table[0, t // 16], :, t % 16, 17] = bad
            c.upload()
            out, lse = c.attend(window=window)
            p = np.arange(L - n, L)
            seen = kv.sees(p, t, window, 0)
            assert self_equal(torch, out[~torch.from_numpy(seen).cuda()], base[~torch.from_numpy(seen).cuda()])
            got = down(out)[seen]
            if name == "v" and fmt != "i8":
                keep = np.arange(128) != 17
                assert np.array_equal(got[..., keep], down(base)[seen][..., keep])
                assert (np.isnan(got[..., 17]) if np.isnan(bad) else got[..., 17] == bad).all()
            elif name == "v" or np.isnan(bad):
                assert not np.isfinite(got).any() or name == "v" and not np.isfinite(got).all(-1).any()
            if name == "v":
                assert np.array_equal(down(lse), down(base_lse))


def test_infinite_scores(g, torch):
    # a key of -inf along a positive query is as good as masked; all of them leave a row of zeros
    c = Case(g, torch, [(2, 40)], fmt="f16", H=1, G=1, D=64, page=8)
    c.q = np.abs(c.q) + 0.5
    c.q = kv.round_to(c.q, "f16")
    for t in range(0, 40, 2):
        c.pool["k"][c.table[0, t // 8], :, t % 8, 3] = -np.inf
    c.upload()
    c.check(*c.attend())
    for t in range(40):
        c.pool["k"][c.table[0, t // 8], :, t % 8, 3] = -np.inf
    c.upload()
    out, lse = c.attend()
    assert (down(out) == 0).all() and (down(lse) == -np.inf).all()


@pytest.mark.parametrize("fmt,type", FORMATS)
@pytest.mark.parametrize("n,L", [(1, 300), (80, 300)])
def test_large_scores(g, torch, fmt, type, n, L):
    """Scores of several hundred, rising and falling along the context: the running maximum moves far and often."""
    c = Case(g, torch, [(n, L)], fmt=fmt, type=type, H=1, G=2, page=16, spread=20.0, seed=7)
    c.q = kv.round_to(c.q * 3, type)
    c.upload()
    c.check(*c.attend())
    c.check(*c.attend(scale=1e-3), scale=1e-3)
    tiny = 2.0 ** -60
    c.check(*c.attend(scale=tiny), scale=tiny)


@pytest.mark.parametrize("power", [-90, -30, 0, 30, 90])
@pytest.mark.parametrize("n", [1, 70])
def test_value_scales_of_any_size(g, torch, power, n):
    """8-bit values far outside fp16's range: bf16 rows of any magnitude."""
    c = Case(g, torch, [(n, 200)], type="bf16", H=1, G=4, page=16, seed=8)
    c.scales["v"] = (c.scales["v"] * np.float32(2.0 ** power)).astype(np.float32)
    # magnitudes grow along the context, so what the sums are held against has to follow
    grow = 2.0 ** (np.arange(200) / 20)
    for t in range(200):
        c.scales["v"][c.table[0, t // 16], :, t % 16] *= np.float32(grow[t])
    c.upload()
    c.check(*c.attend())


@pytest.mark.parametrize("power", [-120, -40, 40, 100])
def test_queries_of_any_size(g, torch, power):
    """bf16 queries far outside fp16's range against an 8-bit cache; the scale brings the scores back."""
    c = Case(g, torch, [(1, 90), (40, 200)], type="bf16", H=1, G=4, page=16, seed=9)
    c.q = c.q * 2.0 ** power
    c.q[0, 0] = 0
    c.upload()
    scale = float(np.float32(2.0 ** -power * 0.1)) if power > -120 else 2.0 ** 110
    c.check(*c.attend(scale=scale), scale=scale)


@pytest.mark.parametrize("layout", ["fused", "heads"])
@pytest.mark.parametrize("n,L", [(1, 90), (70, 150)])
def test_strided_queries_and_outputs(g, torch, layout, n, L):
    c = Case(g, torch, [(n, L), (n, L + 3)], page=16, seed=10).upload()
    x, q = rows_of(torch, np.random.default_rng(11), c.rows, c.heads, c.D, "f16", layout)
    c.q = x
    if layout == "fused":
        wide = torch.full((c.rows, c.heads * c.D + 64), 5.0, dtype=torch.float16, device="cuda")
        out = wide[:, 32:32 + c.heads * c.D].view(c.rows, c.heads, c.D)
    else:
        out = torch.empty((c.heads, c.rows, c.D), dtype=torch.float16, device="cuda").permute(1, 0, 2)
    lse = torch.empty((c.rows, c.heads), device="cuda")
    got = g.grinqh_attend(c.desc, c.cache, c.batch, q, out=out, lse=lse)
    assert got.data_ptr() == out.data_ptr()
    c.check(out, lse)
    if layout == "fused":
        assert (wide[:, :32] == 5).all() and (wide[:, -32:] == 5).all()


def test_a_broadcast_query(g, torch):
    c = Case(g, torch, [(6, 50)], page=16).upload()
    one = up(torch, c.q[:1, :1], "f16")
    c.q = np.broadcast_to(c.q[:1, :1], c.q.shape)
    c.check(*c.attend(q=one.expand(c.q.shape)))


def test_no_rows_and_no_sequences(g, torch):
    c = Case(g, torch, [(0, 5), (0, 0)]).upload()
    out = g.grinqh_attend(c.desc, c.cache, c.batch, torch.empty((0, c.heads, c.D), dtype=torch.float16, device="cuda"))
    assert out.shape == (0, c.heads, c.D)
    empty = g.KvBatch(c.batch.block_table[:0], c.batch.seq_lens[:0], c.batch.row_offsets[:1])
    q = torch.ones((3, c.heads, c.D), dtype=torch.float16, device="cuda")
    g.grinqh_attend(c.desc, c.cache, empty, q)
    k, v = g.grinqh_kv_read(c.desc, c.cache, c.batch, 0)
    g.grinqh_kv_write(c.desc, c.cache, c.batch, k, v)


def test_results_are_reproducible(g, torch):
    c = Case(g, torch, [(1, 9000), (200, 3000)], H=2, page=32).upload()
    first = [t.clone() for t in c.attend()]
    for _ in range(3):
        again = c.attend()
        assert self_equal(torch, again[0], first[0]) and torch.equal(again[1], first[1])


def test_other_stream(g, torch):
    """Outputs and workspace made by the binding while the work runs on a stream of its own."""
    c = Case(g, torch, [(1, 9000), (1, 400)], H=2, page=32).upload()
    q = up(torch, c.q, "f16")
    want = c.attend(lse=False)[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    outs = []
    for _ in range(4):
        outs.append(g.grinqh_attend(c.desc, c.cache, c.batch, q, stream=side))
        junk = torch.full((1 << 20,), float("nan"), device="cuda")   # may take over what was freed too early
    side.synchronize()
    for out in outs:
        assert self_equal(torch, out, want)
    del junk


@pytest.mark.parametrize("fmt,type", [("i8", "f16"), ("bf16", "bf16")])
def test_decode_steps_in_a_graph(g, torch, fmt, type):
    """write and attend captured once; the lengths on the device move on between the replays."""
    L0, steps = 70, 6
    c = Case(g, torch, [(1, L0), (1, L0 + 3000)], fmt=fmt, type=type, H=2, page=16, spare=8)
    need = c.width + 1
    table = np.full((2, need), -1, np.int32)
    free = [i for i in range(c.n_pages) if i not in set(c.table[0, :5]) | set(c.table[1])]
    table[0, :5], table[0, 5], table[1, :c.width] = c.table[0, :5], free[0], c.table[1]
    table[1, c.width] = free[1]
    c.table, c.width = table, need
    c.upload()
    rng = np.random.default_rng(12)
    new = [[rows_of(torch, rng, 2, 2, 128, type, "plain") for _ in "kvq"] for _ in range(steps)]
    q = torch.empty((2, c.heads, 128), dtype=dtype(torch, type), device="cuda")
    k, v = [torch.empty((2, 2, 128), dtype=dtype(torch, type), device="cuda") for _ in "kv"]
    out, lse = torch.empty_like(q), torch.empty((2, c.heads), device="cuda")
    bounds = dict(max_rows=1, max_len=L0 + 3000 + steps)
    ws = torch.empty(g.grinqh_attend_workspace_bytes(c.desc, c.heads, 2, 2, **bounds), dtype=torch.uint8, device="cuda")

    def step():
        c.batch.seq_lens.add_(1)
        g.grinqh_kv_write(c.desc, c.cache, c.batch, k, v)
        g.grinqh_attend(c.desc, c.cache, c.batch, q, out=out, lse=lse, workspace=ws, **bounds)

    graph = torch.cuda.CUDAGraph()
    saved = [t.clone() for t in (c.cache.k, c.cache.v)]
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    assert torch.equal(c.cache.k, saved[0]) and torch.equal(c.cache.v, saved[1])   # nothing ran yet
    for i in range(steps):
        k.copy_(new[i][0][1])
        v.copy_(new[i][1][1])
        x = kv.round_to(rng.standard_normal(c.q.shape), type)
        q.copy_(up(torch, x, type))
        graph.replay()
        torch.cuda.synchronize()
        c.lens, c.q = c.lens + 1, x
        for j, name in enumerate("kv"):
            kv.write(c.pool[name], c.scales[name], fmt, c.table, c.lens, c.offsets, new[i][j][0])
        assert c.batch.seq_lens.tolist() == c.lens.tolist()
        c.check(out, lse)


def test_refusals_of_the_binding(g, torch):
    c = Case(g, torch, [(4, 9)], page=16).upload()
    q = up(torch, c.q, "f16")
    with pytest.raises(g.GrinqhError) as e:
        g.grinqh_attend(c.desc, c.cache, c.batch, q.bfloat16()[:, :7], scale=1.0)
    assert e.value.status == g.GRINQH_EINVAL          # 7 query heads over 2
    with pytest.raises(TypeError):
        g.grinqh_attend(c.desc, c.cache, c.batch, q.int())
    with pytest.raises(g.GrinqhError) as e:
        g.grinqh_attend(c.desc, c.cache, c.batch, q.float())
    assert e.value.status == g.GRINQH_EUNSUPPORTED
    with pytest.raises(ValueError):
        g.grinqh_attend(c.desc, c.cache, c.batch, q[..., :64])
    with pytest.raises(ValueError):
        g.grinqh_attend(c.desc, c.cache, c.batch, q.transpose(1, 2).contiguous().transpose(1, 2))
    with pytest.raises(ValueError):
        g.grinqh_attend(c.desc, c.cache, c.batch, q.cpu())
    with pytest.raises(ValueError):
        g.grinqh_attend(c.desc, c.cache, g.KvBatch(c.batch.block_table, c.batch.seq_lens, c.batch.row_offsets[:1]), q)
    with pytest.raises(ValueError):
        g.grinqh_attend(c.desc, c.cache, c.batch, q, lse=torch.empty((4, 7), device="cuda"))
    with pytest.raises(TypeError):
        g.grinqh_attend(c.desc, c.cache._replace(k=c.cache.k.float()), c.batch, q)
    with pytest.raises(g.GrinqhError) as e:
        g.grinqh_attend(c.desc, c.cache._replace(k_scale=None), c.batch, q)
    assert e.value.status == g.GRINQH_EINVAL
    with pytest.raises(ValueError):
        g.grinqh_kv_write(c.desc, c.cache, c.batch, q[:, :2], q[:, :3])
    with pytest.raises(g.GrinqhError) as e:      # a base that is not 16-byte aligned
        wide = torch.zeros((4, 2 * 128 + 8), dtype=torch.float16, device="cuda")
        g.grinqh_kv_write(c.desc, c.cache, c.batch, wide[:, 1:257].view(4, 2, 128), wide[:, 1:257].view(4, 2, 128))
    assert e.value.status == g.GRINQH_EINVAL
    with pytest.raises(g.GrinqhError) as e:      # outputs that overlap
        g.grinqh_attend(c.desc, c.cache, c.batch, q, out=q[:1].expand(4, 8, 128))
    assert e.value.status == g.GRINQH_EINVAL
    big = Case(g, torch, [(1, 9000)], page=16).upload()
    need = g.grinqh_attend_workspace_bytes(big.desc, big.heads, 1, 1, max_rows=1, max_len=9000)
    if need:
        with pytest.raises(g.GrinqhError) as e:
            big.attend(max_rows=1, max_len=9000, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
        assert e.value.status == g.GRINQH_ESIZE
