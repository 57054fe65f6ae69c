"""Attention over a cache of 8-bit codes against the fp64 oracle, which gets the values that the codes stand for.

Bounds, derived from the arithmetic (u = 2^-24; a rounding to bf16 is off by 2^-8 of a value at most, to fp16 by 2^-11):
  score      codes enter exactly.  Queries of bf16 are fp16 numbers times a power of two, fp32 ones two of them with 2^-22 of a value left,
             and both lose what is below 2^-39 of the largest of 32 rows, and below 2^-29 of their own row's.  A matrix instruction adds 16 or 32 products to its sum with an
             error of up to 3 units of the largest partial sum (6 u; measured), and a product of d terms takes 2 d / 16 of them at
             most: within (d + 4) 2 u sum |q_c k_c|.  Scales, cap, bias and the change to base 2 add a few roundings of the score (and, in
             bf16 outputs only, 4 u cap from the short form of tanh)
  weight     exp turns the error of a score (and of the maximum) into a relative one; sums add n u
  output     sum_j w_j |v_j| times that and the products with scales (6 u); weights enter as one fp16 term (2^-11) or two (2^-22), and not
             below 2^-36 of the largest scale times its largest code: n 2^-35 of the largest value.  2^-8 |out| for the last rounding
"""
import numpy as np
import pytest

from oracle import bwla_attention_oracle as orc
from oracle import bwla_cache8_oracle as orc8

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def A():
    pytest.importorskip("torch")                       # (in front of the library: one HIP runtime for both)
    from paper_2605_00422_amd import attention_binding
    attention_binding.load()
    return attention_binding


class Case:
    """Sequences in pages of codes: lens cached tokens, of which the last news are new.  Storage that no table names and pages that do not
    exist hold NaN codes (e4m3) or anything (i8) under scales of NaN; so do pages all of whose tokens are in nan_tokens."""

    def __init__(self, code, dtype, d, hq, hkv, page, lens, news, seed=0, gone=(), order="heads", one_new=False, spare=2, nan_tokens=(), spread=1.0):
        import torch
        self.torch, self.code, self.dtype, self.d, self.hq, self.hkv, self.page, self.lens, self.news = torch, code, dtype, d, hq, hkv, page, lens, news
        rng = np.random.default_rng(seed)
        T = self.T = torch.bfloat16 if dtype == "bf16" else torch.float32
        n, per = len(lens), max(1, max(-(-x // page) for x in lens))
        self.pages = n * per + spare
        table = rng.permutation(self.pages)[:n * per].reshape(n, per).astype(np.int32)
        junk = lambda: rng.integers(0, 256, (self.pages, hkv, page, d)).astype(np.uint8) if code == "i8" else np.full((self.pages, hkv, page, d), 0x7f, np.uint8)  # noqa: E731
        raw, scale = [junk(), junk()], [np.full((self.pages, hkv), np.nan, np.float32) for _ in range(2)]
        self.kv, self.exists = [], []
        for b, m in enumerate(lens):
            self.exists.append([(b, j // page) not in gone for j in range(m)])
            both = [np.zeros((m, hkv, d)), np.zeros((m, hkv, d))]
            for e in range(-(-m // page)):
                if (b, e) in gone:
                    continue
                p, j0 = table[b, e], e * page
                j1 = min(m, j0 + page)
                for i in range(2):
                    x = rng.standard_normal((j1 - j0, hkv, d)) * np.exp(spread * rng.standard_normal((1, hkv, 1)))
                    for h in range(hkv):
                        s = np.float32(np.abs(x[:, h]).max() / orc8.TOP[code])
                        c = orc8.nearest(code, x[:, h] / np.float64(s))
                        dead = [j for j in range(j0, j1) if (b, j) in nan_tokens]
                        as_bytes = torch.from_numpy(c).to(torch.int8 if code == "i8" else torch.float8_e4m3fn).view(torch.uint8).numpy()
                        if code != "i8":
                            as_bytes[[j - j0 for j in dead]] = 0xff
                        raw[i][p, h, :j1 - j0] = as_bytes
                        scale[i][p, h] = np.nan if len(dead) == j1 - j0 else s
                        both[i][j0:j1, h] = c * np.float64(s)
            self.kv.append(both)
        for b, p in gone:
            table[b, p] = -1 if (b + p) % 2 else self.pages + 7
        self.table_np = table
        as_code = torch.int8 if code == "i8" else torch.float8_e4m3fn
        k, v = (torch.from_numpy(x) for x in raw)
        if order == "tokens":                          # (page, slot, head, column) in memory
            k, v = (x.transpose(1, 2).contiguous().cuda().transpose(1, 2) for x in (k, v))
        elif order == "both":                          # keys and values of a page side by side, rows 48 bytes apart
            both = torch.full((self.pages, 2, hkv, page, d + 48), 0x7f, dtype=torch.uint8)
            both[:, 0, ..., :d], both[:, 1, ..., :d] = k, v
            both = both.cuda()
            k, v = both[:, 0, ..., :d], both[:, 1, ..., :d]
        else:
            k, v = k.cuda(), v.cuda()
        self.k, self.v = k.view(as_code), v.view(as_code)
        wide = [torch.full((self.pages, hkv + 3), float("nan")) for _ in range(2)]
        for w, s in zip(wide, scale):
            w[:, :hkv] = torch.from_numpy(s)
        self.ks, self.vs = (w.cuda()[:, :hkv] for w in wide)
        self.tokens = sum(news)
        self.q = torch.from_numpy((1.5 * rng.standard_normal((self.tokens, hq, d))).astype(np.float32)).to(T)
        i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32).cuda()  # noqa: E731
        self.i32, self.table, self.length = i32, i32(table), i32(lens)
        self.first = None if one_new else i32(np.concatenate([[0], np.cumsum(news)]))

    def cache(self, A):
        return A.KVCache8(self.k, self.v, self.ks, self.vs, self.T)

    def batch(self, A, **kw):
        d = dict(tokens=self.tokens, max_new=max(self.news), max_len=max(self.lens))
        return A.Batch(self.table, self.length, self.first, **{**d, **kw})

    def options(self, rng, names):
        """(keyword arguments of Score, a function of the sequence: those of the oracle)."""
        n, m = len(self.lens), max(max(self.lens), 1)
        kw, per = {}, {}
        if "cap" in names:
            kw["cap"] = 5.0
        if "cap of 50" in names:
            kw["cap"] = 50.0
        if "window of 2" in names:
            kw["window"] = 2
        if "high cap" in names:
            kw["cap"] = 200.0
        if "slopes" in names:
            kw["slopes"] = self.torch.tensor([0.3 / (h + 1) for h in range(self.hq)], dtype=self.torch.float32).cuda()
        if "window" in names:
            kw["window"] = 37
        if "prefix" in names:
            per["prefix"] = rng.integers(0, m, n)
        if "doc" in names:
            per["doc"] = rng.integers(-1, 3, (n, m))
        if "runs" in names:
            per["doc"] = np.sort(rng.integers(0, 4, (n, m)), axis=1)
        if "position" in names:
            per["position"] = np.cumsum(rng.integers(1, 4, (n, m)), axis=1)
        dev = {k: self.i32(v) for k, v in per.items()}

        def oracle(b):
            o = {k: v for k, v in kw.items() if k != "slopes"}
            if "slopes" in kw:
                o["slopes"] = kw["slopes"].cpu().numpy()
            o.update({k: (int(min(v[b], self.lens[b])) if k == "prefix" else v[b]) for k, v in per.items()})
            return o
        return {**kw, **dev}, oracle


def call(c, A, kw, scale=None, q=None, batch=None):
    torch = c.torch
    cache, batch, q = c.cache(A), batch or c.batch(A), c.q.cuda() if q is None else q
    out = torch.full((q.shape[0], c.hq, c.d), float("nan"), dtype=c.T, device="cuda")
    lse = torch.full((q.shape[0], c.hq), float("nan"), device="cuda")
    ws = torch.full((max(16, A.attention8_workspace_size(cache, batch, c.hq)),), 0xff, dtype=torch.uint8, device="cuda")
    A.attention8_forward(cache, batch, A.Score(c.d ** -0.5 if scale is None else scale, **kw), q, out, lse, ws)
    return out, lse


def check(c, A, names=(), seed=1, own=False, few=False):
    """own: what is lost is relative to each row's own largest element, not to all rows'.  few: rows see few keys, of scores below 0.6 of
    the cap: then tanh is off by 4 u of itself, as scales and products are, and nothing by units of the cap."""
    torch = c.torch
    kw, per = c.options(np.random.default_rng(seed), names)
    scale = c.d ** -0.5
    out, lse = call(c, A, kw)
    got, lse = out.float().cpu().numpy(), lse.cpu().numpy()
    row, bf = 0, c.dtype == "bf16"
    for b, (n, new) in enumerate(zip(c.lens, c.news)):
        o = per(b)
        k, v = c.kv[b]
        rows = slice(row, row + new)
        q = c.q[rows].double().numpy()
        out_b, lse_b, _, vabs, qk, top = orc.attend(q, k, v, scale, exists=c.exists[b], **o)
        row += new
        cap = o.get("cap", 0.0)
        if few:
            assert cap and np.max(np.where(np.isfinite(top), top, 0)) < 0.5 * cap
            cap = 0.0
        lost = 2.0 ** -38 * c.d * (np.abs(c.q.double().numpy()).max() if new else 0) * (np.abs(k).max() if n else 0) * scale
        if own:
            lost = 2.0 ** -28 * c.d * np.abs(q).max(-1) * np.abs(k).max() * scale
        eps = 2 * (c.d + 4) * U * qk + 8 * U * (top + cap) + (8 * U * cap if bf else 0) + lost
        rel = np.expm1(np.minimum(2 * eps, 80.0)) + (2 * n + 24) * U
        bound = vabs * (rel[..., None] + (2.0 ** -11 if bf else 2.0 ** -22)) + np.abs(out_b) * (2.0 ** -8 if bf else 4 * U)
        bound = bound + n * 2.0 ** -35 * (np.abs(v).max() if n else 0) + 1e-30
        if own:                                        # (scores off by more than 1 / 2 say nothing, but both are means of the values)
            bound = bound + np.where(eps > 0.5, 2.5 * np.abs(v).max(), 0.0)[..., None]
        assert np.all(np.abs(got[rows] - out_b) <= bound), (b, np.max(np.abs(got[rows] - out_b) / bound))
        empty = np.isneginf(lse_b)
        assert np.array_equal(np.isneginf(lse[rows]), empty)
        ok = ~empty
        assert np.all(np.abs(lse[rows][ok] - lse_b[ok]) <= (rel + 8 * U * (np.abs(np.where(ok, lse_b, 0)) + 1))[ok]), b
    return out


LAYOUTS = [("bf16", 128, 8, 2, 16), ("bf16", 64, 4, 4, 16), ("bf16", 80, 6, 2, 8), ("bf16", 256, 5, 1, 32), ("bf16", 16, 3, 3, 64),
           ("f32", 128, 4, 2, 16), ("f32", 64, 2, 2, 8), ("f32", 48, 7, 1, 16), ("f32", 256, 2, 1, 16), ("f32", 144, 2, 2, 32), ("bf16", 144, 24, 1, 16)]
LENGTHS = [  # (cached, new): one token; chunks; whole prompts; lengths of zero and one; block and tile edges
    ([1, 33, 0, 300, 32], [1, 1, 1, 1, 1]),
    ([257, 64, 1, 65], [3, 2, 1, 5]),
    ([130, 63, 1, 0, 97], [130, 63, 1, 0, 33]),
]
CODES = ["i8", "e4m3"]


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("lens,news", LENGTHS)
@pytest.mark.parametrize("layout", LAYOUTS)
def test_layouts_and_lengths(A, code, layout, lens, news):
    check(Case(code, *layout, lens, news, seed=5, one_new=set(news) == {1}), A)


@pytest.mark.parametrize("names", [("cap",), ("high cap",), ("slopes",), ("window",), ("prefix",), ("doc",), ("runs",), ("position",),
                                   ("cap", "slopes", "position"), ("window", "prefix"), ("window", "position", "doc"),
                                   ("cap", "slopes", "window", "prefix", "doc", "position")])
@pytest.mark.parametrize("code,dtype", [("i8", "bf16"), ("e4m3", "bf16"), ("i8", "f32"), ("e4m3", "f32")])
@pytest.mark.parametrize("lens,news", [([200, 70], [1, 1]), ([300, 41], [4, 3]), ([190, 260], [190, 70])])
def test_masks_caps_and_biases(A, code, dtype, lens, news, names):
    check(Case(code, dtype, 64, 6, 2, 16, lens, news, seed=9), A, names)


@pytest.mark.parametrize("names", [("slopes",), ("slopes", "prefix"), ("slopes", "window", "runs"), ("slopes", "prefix", "doc"), ("slopes", "position")])
@pytest.mark.parametrize("code,dtype,page", [("i8", "bf16", 64), ("e4m3", "f32", 16)])
@pytest.mark.parametrize("lens,news", [([700, 333], [650, 90]), ([500, 64], [2, 1])])
def test_a_bias_without_a_cap(A, code, dtype, page, lens, news, names):
    """Keys in front of every row, among the rows and, in prefixes, behind them."""
    check(Case(code, dtype, 128, 6, 2, page, lens, news, seed=17), A, names)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("lens,news,names", [([5, 2, 1], [1, 1, 1], ("cap of 50",)), ([400, 37], [1, 1], ("cap of 50", "window of 2")),
                                             ([300, 90], [300, 70], ("cap of 50", "window of 2"))])
def test_caps_of_rows_that_see_few_keys(A, code, dtype, lens, news, names):
    """Their scores and lse keep their bits: a cap far above them costs none."""
    check(Case(code, dtype, 64, 6, 2, 16, lens, news, seed=19, spread=0.2), A, names, few=True)


@pytest.mark.parametrize("new", [1, 9, 60])
@pytest.mark.parametrize("code,dtype", [("i8", "bf16"), ("e4m3", "f32")])
def test_pages_that_do_not_exist(A, code, dtype, new):
    gone = {(0, 0), (0, 3), (1, 0), (1, 1), (1, 2), (1, 3), (1, 4), (1, 5), (2, 5)}
    check(Case(code, dtype, 128, 8, 4, 16, [120, 90, 96], [new] * 3, gone=gone), A)
    check(Case(code, dtype, 128, 8, 4, 16, [120, 90, 96], [new] * 3, gone=gone), A, ("prefix", "window"))


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 3, 70])
def test_tokens_that_no_query_sees_may_hold_anything(A, code, dtype, new):
    """Single tokens of NaN codes, and whole pages of them under scales of NaN."""
    import torch
    dead = {(0, 5), (0, 64), (0, 77), (1, 0), (1, 70)} | {(0, j) for j in range(16, 32)} | {(1, j) for j in range(48, 64)}
    c = Case(code, dtype, 64, 4, 2, 16, [200, 150], [new, new], nan_tokens=dead)
    doc = np.zeros((2, 200), np.int32)
    for b, j in dead:
        doc[b, j] = -1 if j % 2 else 7 + j             # in none, or in one of its own
    c.options = lambda rng, names: ({"doc": c.i32(doc)}, lambda b: {"doc": doc[b]})
    out = check(c, A)
    assert torch.isfinite(out.float()).all()


@pytest.mark.parametrize("order", ["tokens", "both"])
@pytest.mark.parametrize("code,dtype", [("i8", "bf16"), ("e4m3", "f32")])
@pytest.mark.parametrize("new", [1, 100])
def test_strides_of_the_cache(A, code, dtype, order, new):
    check(Case(code, dtype, 64, 8, 4, 16, [130, 111], [new, new], order=order), A)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 90])
def test_queries_apart_and_rows_of_no_sequence(A, dtype, new):
    import torch
    c = Case("i8", dtype, 64, 4, 2, 16, [120, 95], [new, new])
    wide = torch.full((2 * new + 5, 4 * 64 + 3 * 64), float("nan"), dtype=c.T, device="cuda")
    q = c.q.cuda()
    wide[2:2 * new + 2, :256] = q.reshape(2 * new, 256)
    rows = wide[:, :256].unflatten(1, (4, 64))
    batch = A.Batch(c.table, c.length, c.i32([2, 2 + new, 2 + 2 * new]), tokens=2 * new + 5, max_new=new, max_len=120)
    cache = c.cache(A)
    ws = torch.empty(max(16, A.attention8_workspace_size(cache, batch, 4)), dtype=torch.uint8, device="cuda")
    out = torch.full((2 * new + 5, 4, 64), 9.0, dtype=c.T, device="cuda")
    A.attention8_forward(cache, batch, A.Score(0.125), rows, out, None, ws)
    want, _ = call(c, A, {}, 0.125)
    assert torch.equal(out[2:2 * new + 2], want)
    assert (out[:2] == 9).all() and (out[2 * new + 2:] == 9).all()


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("news", [[5, 3], [200, 9]])
def test_more_new_tokens_than_cached_ones(A, code, news):
    check(Case(code, "bf16", 64, 4, 2, 16, [3, 2], news), A)


@pytest.mark.parametrize("lens,news", [([3000, 900], [1, 1]), ([2100, 5000], [7, 2])])
@pytest.mark.parametrize("code,dtype", [("i8", "bf16"), ("e4m3", "bf16"), ("i8", "f32")])
def test_long_caches_are_split_and_joined(A, code, dtype, lens, news):
    c = Case(code, dtype, 128, 8, 1, 64, lens, news)
    out = check(c, A)
    assert c.torch.equal(out, check(c, A))
    check(c, A, ("window", "prefix", "cap"))


MANY_ROWS = [  # (layout, cached, new): few workgroups, so that the cached tokens are dealt out over several and their parts added up
    (("bf16", 128, 4, 2, 16), [1500, 40, 0, 700], [80, 40, 0, 33]),
    (("bf16", 80, 6, 2, 8), [1100, 257], [70, 257]),
    (("bf16", 256, 8, 1, 32), [900], [60]),
    (("f32", 128, 4, 2, 16), [900, 513], [50, 51]),
    (("f32", 48, 7, 1, 16), [520], [300]),
]


@pytest.mark.parametrize("names", [(), ("cap", "slopes"), ("window", "prefix"), ("runs",), ("doc",), ("window", "position")])
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("layout,lens,news", MANY_ROWS)
def test_many_rows_over_parts_of_the_cache(A, code, layout, lens, news, names):
    c = Case(code, *layout, lens, news, seed=21)
    assert A.attention8_workspace_size(c.cache(A), c.batch(A), c.hq) > 0
    out = check(c, A, names)
    assert c.torch.equal(out, check(c, A, names))


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("new", [1, 100])
@pytest.mark.parametrize("spread", [3.0, 6.0])
def test_scales_of_very_different_pages(A, code, new, spread):
    """Scales that differ by e^(spread times a few) from page to page, keys and values alike."""
    c = Case(code, "f32", 64, 4, 2, 16, [400, 90], [new] * 2 if new == 1 else [new, 90], seed=31, spread=spread)
    c.q *= float(np.exp(-2 * spread))
    check(c, A)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,news", [([500], [500]), ([3000], [2]), ([1500], [100])])
def test_scores_that_rise_along_the_cache(A, dtype, lens, news):
    """Each key's product with every query is larger than the one before it by enough to move the maximum again and again."""
    import torch
    c = Case("i8", dtype, 64, 4, 2, 16, lens, news, seed=24)
    n = lens[0]
    k = np.zeros((n, 2, 64))
    for e in range(-(-n // 16)):                       # a page's first column rises as its scale does
        p, j = c.table_np[0, e], np.arange(e * 16, min(n, e * 16 + 16))
        codes = np.clip(np.rint(60.0 * (j + 1) / n / (60.0 * (e + 1) * 16 / n) * 127), -127, 127)
        s = np.float32(60.0 * (e + 1) * 16 / n / 127)
        c.k[int(p), :, :len(j), 0] = torch.from_numpy(codes.astype(np.int8)).cuda()
        c.ks[int(p)] = float(s)
        own = c.k[int(p), :, :len(j)].cpu().double().numpy().transpose(1, 0, 2)
        k[j] = own * np.float64(s)
    c.kv[0][0] = k
    c.q[:, :, 0] = 8.0
    check(c, A)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 100])
@pytest.mark.parametrize("size", [1e-30, 1e-6, 1e6, 1e30])
def test_queries_of_very_small_and_very_large_values(A, dtype, new, size):
    c = Case("i8", dtype, 64, 4, 2, 16, [300], [new], seed=3)
    c.q = (c.q.double() * size).to(c.T)
    scale = 1.0 / size / 8
    if not 1e-37 < scale < 1e37:
        pytest.skip("not a scale")
    out, _ = call(c, A, {}, scale)
    want = orc.attend(c.q.double().numpy(), *c.kv[0], np.float64(np.float32(scale)))[0]
    err = np.abs(out.double().cpu().numpy() - want).max() / np.abs(want).max()
    assert err <= (2.0 ** -7 if dtype == "bf16" else 1e-4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("new", [3, 100])
@pytest.mark.parametrize("size,names", [(2.0 ** 20, ()), (2.0 ** 100, ()), (2.0 ** -50, ()), (2.0 ** 40, ("cap", "doc")), (2.0 ** 30, ("slopes", "window"))])
def test_a_row_of_another_size_takes_nothing_from_the_others(A, code, dtype, new, size, names):
    """One head of a token (and, of 100, a second one, and one of zeros) has queries of another magnitude than the rows beside it."""
    c = Case(code, dtype, 64, 4, 2, 16, [300], [new], seed=12)
    c.q[1, 2] *= size
    if new > 50:
        c.q[40, 1] *= size ** 0.5
        c.q[41, 1] = 0
    out = check(c, A, names, own=True)
    assert c.torch.isfinite(out.float()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("new", [2, 70])
def test_rows_of_nan_stay_their_own(A, code, dtype, new):
    """A query that is NaN makes NaN of its row and of no other; one that sees nothing gives 0 whatever it holds."""
    import torch
    c = Case(code, dtype, 64, 4, 2, 16, [200, 90], [new, new], seed=3)
    want, lse0 = call(c, A, {})
    bad = c.q.clone()
    bad[1, 2, 7] = float("nan")
    out, lse = call(c, A, {}, q=bad.cuda())
    assert torch.isnan(out[1, 2].float()).all() and torch.isnan(lse[1, 2])
    same = torch.ones(2 * new, 4, dtype=torch.bool, device="cuda")
    same[1, 2] = False
    assert torch.equal(out[same], want[same]) and torch.equal(lse[same], lse0[same])
    doc = np.zeros((2, 200), np.int32)
    doc[0, 200 - new + 1] = -1                          # row 1 sees nothing
    out, lse = call(c, A, {"doc": c.i32(doc)}, q=bad.cuda())
    assert not out[1].any() and torch.isneginf(lse[1]).all() and torch.isfinite(out.float()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 90])
def test_one_key_and_equal_values(A, dtype, new):
    """A row that sees one key is that key's value, and a mean of equal values is their value."""
    import torch
    c = Case("i8", dtype, 64, 4, 4, 16, [100], [new], seed=6)
    doc = np.arange(100)[None].astype(np.int32)         # every token sees itself alone
    out, _ = call(c, A, {"doc": c.i32(doc)})
    want = torch.from_numpy(c.kv[0][1][100 - new:].astype(np.float32))
    near = 2.0 ** -8 if dtype == "bf16" else 4 * U     # (weights are 1 and codes exact, but scales differ from the largest of a block by fp16's rounding)
    assert ((out.float().cpu() - want).abs() <= (near + (2.0 ** -11 if dtype == "bf16" else 2.0 ** -21)) * want.abs() + 1e-6).all()


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("new", [1, 17])
def test_pages_beyond_32_bits(A, code, new):
    import torch
    hkv, page, d = 8, 64, 128
    pages = (1 << 32) // (hkv * page * d) + 40
    small = Case(code, "bf16", d, 16, hkv, page, [150, 200], [new, new], one_new=new == 1)
    want, _ = call(small, A, {})
    T = small.k.dtype
    k = torch.zeros(pages, hkv, page, d, dtype=torch.uint8, device="cuda")
    v, ks, vs = torch.zeros_like(k), torch.zeros(pages, hkv, device="cuda"), torch.zeros(pages, hkv, device="cuda")
    far = np.array([[pages - 1, 0, pages - 20, 5], [pages - 7, 1, pages - 2, pages - 3]], np.int32)
    for b in range(2):
        for i, p in enumerate(small.table_np[b]):
            k[far[b, i]], v[far[b, i]] = small.k.view(torch.uint8)[p], small.v.view(torch.uint8)[p]
            ks[far[b, i]], vs[far[b, i]] = small.ks[p], small.vs[p]
    small.k, small.v, small.ks, small.vs, small.table = k.view(T), v.view(T), ks, vs, small.i32(far)
    assert torch.equal(call(small, A, {})[0], want)


@pytest.mark.parametrize("new", [1, 100])
def test_captured_and_replayed_beside_eager_calls(A, new):
    import torch
    c = Case("i8", "bf16", 128, 8, 2, 16, [900, 300], [new, new], seed=2)
    cache, batch, score = c.cache(A), c.batch(A), A.Score(c.d ** -0.5)
    q = c.q.cuda()
    need = max(16, A.attention8_workspace_size(cache, batch, 8))
    ws, other = (torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(2))
    out, eager = torch.empty_like(q), torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        A.attention8_forward(cache, batch, score, q, out, None, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        A.attention8_forward(cache, batch, score, q, out, None, ws)
    for i in range(4):
        q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(i)).to(q.dtype))
        out.fill_(7)
        graph.replay()
        A.attention8_forward(cache, batch, score, q, eager, None, other)
        torch.cuda.synchronize()
        assert torch.equal(out, eager)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 100])
@pytest.mark.parametrize("scale", [0.0, 1e-44, 1e-39, 1e30])
def test_scales_of_values_at_the_edges_of_fp32(A, dtype, new, scale):
    import torch
    c = Case("i8", dtype, 64, 4, 2, 16, [150], [new], seed=4)
    c.vs[c.vs == c.vs] = scale
    out, lse = call(c, A, {})
    k = c.kv[0][0]
    codes = torch.cat([c.v[int(p)].transpose(0, 1) for p in c.table_np[0]])[:150].double().cpu().numpy()
    want = orc.attend(c.q.double().numpy(), k, codes * np.float64(np.float32(scale)), c.d ** -0.5)[0]
    assert torch.isfinite(lse).all()
    # (below 2^-126 outputs are numbers of few bits: half a unit of bf16's or fp32's smallest, and one that products lose)
    tiny = 2.0 ** -133 * 1.01 if dtype == "bf16" else 2.0 ** -148
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= np.abs(want).max() * (2.0 ** -7 if dtype == "bf16" else 1e-5) + tiny)


@pytest.mark.parametrize("new", [1, 100])
def test_large_queries_small_keys_and_a_large_scale(A, new):
    """Factors whose product in another order would leave fp32's range."""
    c = Case("i8", "f32", 64, 4, 2, 16, [150], [new], seed=4)
    c.q *= 1e30
    c.ks *= 1e-36
    c.kv[0][0] = c.kv[0][0] * 1e-36
    out, _ = call(c, A, {}, 1e5)
    want = orc.attend(c.q.double().numpy(), c.kv[0][0], c.kv[0][1], np.float64(np.float32(1e5)))[0]
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= 1e-4 * np.abs(want).max())
