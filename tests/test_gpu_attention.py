"""The cache, rotation, attention and eviction kernels against the fp64 oracle, at the sizes and masks where they can go wrong.

Bounds, derived from the arithmetic (u = 2^-24; a rounding to bf16 is off by 2^-8 of a value at most, 2^-9 in the mean):
  score      a product of d terms in fp32 has an error of (d + 4) u sum |q_c k_c| at most; scaling, cap, bias and the change to
             base 2 add a few roundings of the score (and, in bf16 outputs only, 4 u cap from the short form of tanh)
  weight     exp turns the error of a score (and of the maximum or lse) into a relative one; sums add n u
  output     sum_j w_j |v_j| times that, plus 2^-9 of it for weights entered as bf16 (their errors have random signs over many
             keys; rows that see few carry 16 bits) and 2^-8 |out| for the last rounding
"""
import numpy as np
import pytest

from oracle import bwla_attention_oracle as orc

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def A():
    pytest.importorskip("torch")                       # (in front of the library: one HIP runtime for both)
    from paper_2605_00422_amd import attention_binding
    attention_binding.load()
    return attention_binding


class Case:
    """Sequences in pages: lens cached tokens, of which the last news are new; storage that no table names, behind the
    lengths and in pages that do not exist is NaN."""

    def __init__(self, dtype, d, hq, hkv, page, lens, news, seed=0, gone=(), order="heads", one_new=False, spare=2, nan_tokens=()):
        import torch
        self.torch, self.dtype, self.d, self.hq, self.hkv, self.page, self.lens, self.news = torch, dtype, d, hq, hkv, page, lens, news
        rng = np.random.default_rng(seed)
        T = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.T = T
        draw = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(T)  # noqa: E731
        n, per = len(lens), max(1, max(-(-x // page) for x in lens))
        self.pages = n * per + spare
        table = rng.permutation(self.pages)[:n * per].reshape(n, per).astype(np.int32)
        self.kv, k, v = [], *(torch.full((self.pages, hkv, page, d), float("nan"), dtype=T) for _ in range(2))
        self.exists = []
        for b, m in enumerate(lens):
            kb, vb = draw(m, hkv, d), draw(m, hkv, d)
            for j in range(m):
                if (b, j) in nan_tokens:
                    kb[j], vb[j] = float("nan"), float("inf")
            self.exists.append([(b, j // page) not in gone for j in range(m)])
            for j in range(m):
                if self.exists[b][j]:
                    k[table[b, j // page], :, j % page], v[table[b, j // page], :, j % page] = kb[j], vb[j]
            self.kv.append((kb, vb))
        for b, p in gone:
            table[b, p] = -1 if (b + p) % 2 else self.pages + 7
        self.table_np = table
        if order == "tokens":                          # (page, slot, head, column) in memory
            k, v = (x.transpose(1, 2).contiguous().cuda().transpose(1, 2) for x in (k, v))
        elif order == "both":                          # keys and values of a page side by side, rows 24 columns apart
            both = torch.full((self.pages, 2, hkv, page, d + 24), float("nan"), dtype=T)
            both[:, 0, ..., :d], both[:, 1, ..., :d] = k, v
            both = both.cuda()
            k, v = both[:, 0, ..., :d], both[:, 1, ..., :d]
        else:
            k, v = k.cuda(), v.cuda()
        self.k, self.v = k, v
        self.tokens = sum(news)
        self.q = (1.5 * draw(self.tokens, hq, d).float()).to(T)
        i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32).cuda()  # noqa: E731
        self.i32, self.table, self.length = i32, i32(table), i32(lens)
        self.first = None if one_new else i32(np.concatenate([[0], np.cumsum(news)]))

    def batch(self, A, **kw):
        d = dict(tokens=self.tokens, max_new=max(self.news), max_len=max(self.lens))
        return A.Batch(self.table, self.length, self.first, **{**d, **kw})

    def options(self, rng, names):
        """(keyword arguments of Score, a function of the sequence: those of the oracle)."""
        n, m = len(self.lens), max(max(self.lens), 1)
        kw, per = {}, {}
        if "cap" in names:
            kw["cap"] = 5.0
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


def check(c, A, names=(), weights=True, seed=1, order=None):
    """attention_forward (and the sums of weights, fused and on their own) against the oracle."""
    torch = c.torch
    rng = np.random.default_rng(seed)
    kw, per = c.options(rng, names)
    scale = c.d ** -0.5
    cache, batch, score = A.KVCache(c.k, c.v), c.batch(A), A.Score(scale, **kw)
    q = c.q.cuda()
    out = torch.full_like(q, float("nan"))
    lse = torch.full((c.tokens, c.hq), float("nan"), device="cuda")
    sums = cache.weights() if weights else None
    ws = torch.full((max(16, A.attention_workspace_size(cache, batch, c.hq, weights)),), 0xff, dtype=torch.uint8, device="cuda")
    A.attention_forward(cache, batch, score, q, out, lse, sums, ws)
    alone = cache.weights() + 2.0
    ws2 = torch.full((max(16, A.attention_weights_workspace_size(cache, batch, c.hq)),), 0xff, dtype=torch.uint8, device="cuda")
    if weights:
        A.attention_weights(cache, batch, score, q, lse, alone, ws2)
    bare = torch.empty_like(out)                       # without the optional outputs: the same
    A.attention_forward(cache, batch, score, q, bare, None, None, ws)
    assert torch.equal(bare, out)
    got, lse = out.float().cpu().numpy(), lse.cpu().numpy()
    row, bf = 0, c.dtype == "bf16"
    want_sums = np.zeros(tuple(c.k.shape[:3]))
    sum_bound = np.zeros_like(want_sums)
    for b, (n, new) in enumerate(zip(c.lens, c.news)):
        o = per(b)
        k, v = (x.float().numpy() for x in c.kv[b])
        rows = slice(row, row + new)
        out_b, lse_b, sums_b, vabs, qk, top = orc.attend(c.q[rows].float().numpy(), k, v, scale, exists=c.exists[b], **o)
        row += new
        cap = o.get("cap", 0.0)
        eps = 2 * (c.d + 4) * U * qk + 8 * U * (top + cap) + (8 * U * cap if bf else 0)
        rel = np.expm1(2 * eps) + (2 * n + 16) * U
        bound = vabs * (rel[..., None] + (2.0 ** -9 if bf else 0)) + np.abs(out_b) * (2.0 ** -8 if bf else 4 * U) + 1e-30
        assert np.all(np.abs(got[rows] - out_b) <= bound), (b, np.max(np.abs(got[rows] - out_b) / bound))
        empty = np.isneginf(lse_b)
        assert np.array_equal(np.isneginf(lse[rows]), empty)
        ok = ~empty
        assert np.all(np.abs(lse[rows][ok] - lse_b[ok]) <= (rel + 8 * U * (np.abs(np.where(ok, lse_b, 0)) + 1))[ok]), b
        for j in range(n):
            if c.exists[b][j]:
                p, s = c.table_np[b, j // c.page], j % c.page
                want_sums[p, :, s] += sums_b[j]
                most = (rel + 8 * U * (np.abs(np.where(ok, lse_b, 0)) + top)).max() if new else 0.0
                sum_bound[p, :, s] = sums_b[j] * (most + (new * c.hq // c.hkv + 8) * U) + 1e-37
    if weights:
        # (fp32 sums that start at 0 and at 2; what underflows in fp32 is 0)
        assert np.all(np.abs(sums.cpu().numpy() - want_sums) <= sum_bound + 1e-35)
        assert np.all(np.abs(alone.cpu().numpy() - 2.0 - want_sums) <= sum_bound + 2 * U * (2.0 + want_sums))
    return out


LAYOUTS = [("bf16", 128, 8, 2, 16), ("bf16", 64, 4, 4, 16), ("bf16", 80, 6, 2, 8), ("bf16", 256, 5, 1, 32), ("bf16", 8, 3, 3, 64),
           ("f32", 128, 4, 2, 16), ("f32", 64, 2, 2, 8), ("f32", 40, 7, 1, 16), ("f32", 256, 2, 1, 16), ("f32", 136, 2, 2, 32), ("bf16", 136, 24, 1, 16)]
LENGTHS = [  # (cached, new): one token; chunks; whole prompts; lengths of zero and one; block and tile edges
    ([1, 33, 0, 300, 32], [1, 1, 1, 1, 1]),
    ([257, 64, 1, 65], [3, 2, 1, 5]),
    ([130, 63, 1, 0, 97], [130, 63, 1, 0, 33]),
]


@pytest.mark.parametrize("lens,news", LENGTHS)
@pytest.mark.parametrize("layout", LAYOUTS)
def test_layouts_and_lengths(A, layout, lens, news):
    check(Case(*layout, lens, news, seed=5, one_new=set(news) == {1}), A)


@pytest.mark.parametrize("names", [("cap",), ("slopes",), ("window",), ("prefix",), ("doc",), ("runs",), ("position",),
                                   ("cap", "slopes", "position"), ("window", "prefix"), ("window", "position", "doc"),
                                   ("cap", "slopes", "window", "prefix", "doc", "position")])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,news", [([200, 70], [1, 1]), ([300, 41], [4, 3]), ([190, 260], [190, 70])])
def test_masks_caps_and_biases(A, dtype, lens, news, names):
    check(Case(dtype, 64, 6, 2, 16, lens, news, seed=9), A, names)


@pytest.mark.parametrize("new", [1, 9, 60])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_that_do_not_exist(A, dtype, new):
    gone = {(0, 0), (0, 3), (1, 0), (1, 1), (1, 2), (1, 3), (1, 4), (1, 5), (2, 5)}
    check(Case(dtype, 128, 8, 4, 16, [120, 90, 96], [new] * 3, gone=gone), A)
    check(Case(dtype, 128, 8, 4, 16, [120, 90, 96], [new] * 3, gone=gone), A, ("prefix", "window"))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 3, 70])
def test_tokens_that_no_query_sees_may_hold_anything(A, dtype, new):
    torch = pytest.importorskip("torch")
    c = Case(dtype, 64, 4, 2, 16, [200, 150], [new, new], nan_tokens={(0, 5), (0, 64), (0, 77), (1, 0), (1, 100)} if new < 70 else {(0, 5), (1, 70)})
    doc = np.zeros((2, 200), np.int32)
    for b, j in ((0, 5), (0, 64), (0, 77), (1, 0), (1, 100), (1, 70)):
        doc[b, j] = -1 if j % 2 else 7 + j           # in none, or in one of its own
    c.options = lambda rng, names: ({"doc": c.i32(doc)}, lambda b: {"doc": doc[b]})
    out = check(c, A)
    assert torch.isfinite(out.float()).all()


@pytest.mark.parametrize("order", ["tokens", "both"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 100])
def test_strides_of_the_cache(A, dtype, order, new):
    check(Case(dtype, 64, 8, 4, 16, [130, 111], [new, new], order=order), A)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 90])
def test_queries_apart_and_rows_of_no_sequence(A, dtype, new):
    import torch
    c = Case(dtype, 64, 4, 2, 16, [120, 95], [new, new])
    cache, score = A.KVCache(c.k, c.v), A.Score(0.125)
    wide = torch.full((2 * new + 5, 4 * 64 + 3 * 64), float("nan"), dtype=c.T, device="cuda")
    q = c.q.cuda()
    wide[2:2 * new + 2, :256] = q.reshape(2 * new, 256)
    rows = wide[:, :256].unflatten(1, (4, 64))
    first = c.i32([2, 2 + new, 2 + 2 * new])           # two rows in front and three behind belong to no sequence
    batch = A.Batch(c.table, c.length, first, tokens=2 * new + 5, max_new=new, max_len=120)
    ws = torch.empty(max(16, A.attention_workspace_size(cache, batch, 4)), dtype=torch.uint8, device="cuda")
    out = torch.full((2 * new + 5, 4, 64), 9.0, dtype=c.T, device="cuda")
    A.attention_forward(cache, batch, score, rows, out, None, None, ws)
    dense, want = c.batch(A), torch.empty_like(q)
    ws = torch.empty(max(16, A.attention_workspace_size(cache, dense, 4)), dtype=torch.uint8, device="cuda")
    A.attention_forward(cache, dense, score, q, want, None, None, ws)
    assert torch.equal(out[2:2 * new + 2], want)
    assert (out[:2] == 9).all() and (out[2 * new + 2:] == 9).all()


@pytest.mark.parametrize("news", [[5, 3], [200, 9]])
def test_more_new_tokens_than_cached_ones(A, news):
    """Rows whose index would be negative see nothing."""
    check(Case("bf16", 64, 4, 2, 16, [3, 2], news), A)


def test_lengths_beyond_the_bounds_are_cut(A):
    import torch
    c = Case("bf16", 64, 4, 2, 16, [100, 64], [1, 1], one_new=True)
    cache, score, q = A.KVCache(c.k, c.v), A.Score(0.125), c.q.cuda()
    outs = []
    for length in (c.i32([100, 64]), c.i32([100, 1 << 30]), c.i32([-5, 64])):
        batch = A.Batch(c.table, length, max_len=100 if len(outs) != 1 else 64)
        out = torch.empty_like(q)
        ws = torch.empty(max(16, A.attention_workspace_size(cache, batch, 4)), dtype=torch.uint8, device="cuda")
        A.attention_forward(cache, batch, score, q, out, None, None, ws)
        outs.append(out)
    assert torch.equal(outs[0][1], outs[1][1]) and not outs[2][0].any() and torch.equal(outs[2][1], outs[0][1])


@pytest.mark.parametrize("new", [1, 17])
def test_pages_beyond_32_bits(A, new):
    """Pages whose bytes lie more than 2^32 behind the first one."""
    import torch
    hkv, page, d = 8, 64, 128
    pages = (1 << 32) // (hkv * page * d * 2) + 40
    k = torch.empty(pages, hkv, page, d, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    small = Case("bf16", d, 16, hkv, page, [150, 200], [new, new], one_new=new == 1)
    far = np.array([[pages - 1, 0, pages - 20, 5], [pages - 7, 1, pages - 2, pages - 3]], np.int32)
    for b in range(2):
        for i, p in enumerate(small.table_np[b]):
            k[far[b, i]], v[far[b, i]] = small.k[p], small.v[p]
    score, q = A.Score(d ** -0.5), small.q.cuda()
    outs, sums = [], []
    for kk, vv, table in ((small.k, small.v, small.table), (k, v, small.i32(far))):
        cache = A.KVCache(kk, vv)
        batch = A.Batch(table, small.length, small.first, tokens=small.tokens, max_new=new, max_len=200)
        ws = torch.empty(max(16, A.attention_workspace_size(cache, batch, 16, True)), dtype=torch.uint8, device="cuda")
        out, lse, w = torch.empty_like(q), torch.empty(small.tokens, 16, device="cuda"), cache.weights()
        A.attention_forward(cache, batch, score, q, out, lse, w, ws)
        outs.append(out)
        sums.append(torch.stack([w[int(p)] for p in table.flatten()]))
    assert torch.equal(*outs) and torch.equal(*sums)


@pytest.mark.parametrize("lens,news", [([3000, 900], [1, 1]), ([2100, 5000], [7, 2])])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_caches_are_split_and_joined(A, dtype, lens, news):
    check(Case(dtype, 128, 8, 1, 64, lens, news), A)
    check(Case(dtype, 128, 8, 1, 64, lens, news), A, ("window", "prefix", "cap"))


MANY_ROWS = [  # (layout, cached, new): few workgroups, so that the cached tokens are dealt out over several and their parts added up
    (("bf16", 128, 4, 2, 16), [1500, 40, 0, 700], [80, 40, 0, 33]),
    (("bf16", 80, 6, 2, 8), [1100, 257], [70, 257]),
    (("bf16", 256, 8, 1, 32), [900], [60]),
    (("f32", 128, 4, 2, 16), [900, 513], [50, 51]),
    (("f32", 40, 7, 1, 16), [520], [300]),
]


@pytest.mark.parametrize("names", [(), ("cap", "slopes"), ("window", "prefix"), ("runs",), ("doc",), ("window", "position"),
                                   ("cap", "slopes", "window", "prefix", "doc", "position")])
@pytest.mark.parametrize("layout,lens,news", MANY_ROWS)
def test_many_rows_over_parts_of_the_cache(A, layout, lens, news, names):
    c = Case(*layout, lens, news, seed=21)
    assert A.attention_workspace_size(A.KVCache(c.k, c.v), c.batch(A), c.hq, False) > 0
    out = check(c, A, names)
    assert c.torch.equal(out, check(c, A, names))


@pytest.mark.parametrize("layout,lens,news", [
    (("bf16", 64, 14, 2, 16), [600], [600]),                                   # rows enough for the other join
    (("f32", 8, 14, 2, 16), [600], [600]),
    (("bf16", 8, 33, 33, 16), [2500, 100, 130, 7], [129, 100, 129, 7]),        # sequences of very different lengths
])
def test_many_rows_joined(A, layout, lens, news):
    c = Case(*layout, lens, news, seed=22)
    assert A.attention_workspace_size(A.KVCache(c.k, c.v), c.batch(A), c.hq, False) > 0
    check(c, A)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,news", [([500], [500]), ([3000], [2]), ([1500], [100])])
def test_scores_that_rise_along_the_cache(A, dtype, lens, news):
    """Each key's product with every query is larger than the one before it by enough to move the maximum again and again."""
    c = Case(dtype, 64, 4, 2, 16, lens, news, seed=24)
    n = lens[0]
    step = c.torch.linspace(0.0, 60.0, n)[:, None]
    k, v = c.kv[0]
    k[:, :, 0] = step.to(c.T)
    c.q[:, :, 0] = 8.0
    for j in range(n):
        c.k[int(c.table_np[0, j // 16]), :, j % 16, 0] = k[j, :, 0].cuda()
    check(c, A)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("names", [(), ("prefix",), ("window",), ("position", "window")])
@pytest.mark.parametrize("run", [1, 5, 40, 200])
def test_rows_of_several_documents(A, dtype, names, run):
    """Short documents, of which many lie in a block, and longer ones, whose ends lie inside a workgroup's rows."""
    class Runs(Case):
        def options(self, rng, names):
            kw, oracle = super().options(rng, names)
            doc = np.stack([(np.arange(max(self.lens)) + 3) // run % 9 for _ in self.lens])
            return {**kw, "doc": self.i32(doc)}, lambda b: {**oracle(b), "doc": doc[b]}
    check(Runs(dtype, 64, 4, 2, 16, [450, 130], [450, 60], seed=23), A, names)


def test_the_same_call_gives_the_same_bits(A):
    import torch
    for lens, news in (([2000, 37], [1, 1]), ([500, 300], [200, 300])):
        c = Case("bf16", 128, 8, 2, 16, lens, news)
        first = check(c, A, ("cap",))
        assert torch.equal(first, check(c, A, ("cap",)))


@pytest.mark.parametrize("lens,news", [([700, 90], [1, 1]), ([150, 200], [150, 80])])
def test_in_a_graph_and_on_another_stream(A, lens, news):
    import torch
    c = Case("bf16", 128, 8, 2, 16, lens, news)
    cache, batch, score = A.KVCache(c.k, c.v), c.batch(A), A.Score(0.1, cap=30.0)
    q = c.q.cuda()
    ws = torch.empty(max(16, A.attention_workspace_size(cache, batch, 8, True)), dtype=torch.uint8, device="cuda")
    out, lse, w = torch.empty_like(q), torch.empty(c.tokens, 8, device="cuda"), cache.weights()

    def step():
        w.zero_()
        A.attention_forward(cache, batch, score, q, out, lse, w, ws)

    step()
    torch.cuda.synchronize()
    want, want_w = out.clone(), w.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    assert torch.equal(out, want) and torch.equal(w, want_w)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(4):
        q.mul_(-1 if i % 2 == 0 else 1)                # eager work between the replays
        g.replay()
        torch.cuda.synchronize()
        got, got_w = out.clone(), w.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, out) and torch.equal(got_w, w)


# ---------------------------------------------------------------- rotation
ROPES = [(64, [32], False), (64, [16], True), (128, [8, 28, 28], False), (128, [5, 40, 19], True), (80, [20], False), (40, [3, 2], False),
         (8, [4], True), (256, [32, 32, 32, 32], False), (96, [0, 48], False), (64, [], False)]


@pytest.mark.parametrize("d,sections,interleaved", ROPES)
@pytest.mark.parametrize("x,dtype", [("f32", "bf16"), ("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
def test_rope_append(A, d, sections, interleaved, x, dtype):
    import torch
    rng = np.random.default_rng(d)
    hq, hkv, page, lens, news = 6, 2, 16, [40, 3, 1, 17], [19, 3, 0, 1]
    c = Case(dtype, d, hq, hkv, page, lens, news)
    pairs, tokens, rows = sum(sections), sum(news), 60
    sections = sections or [0]
    angle = rng.uniform(-np.pi, np.pi, (rows, pairs))
    cos, sin = (torch.from_numpy(f(angle).astype(np.float32)).cuda() for f in (np.cos, np.sin))
    pos = rng.integers(0, rows, (len(sections), tokens)).astype(np.int32)
    T = torch.bfloat16 if x == "bf16" else torch.float32
    width = (hq + 2 * hkv) * d
    wide = torch.from_numpy(rng.standard_normal((tokens, width + 16)).astype(np.float32)).to(T).cuda()
    qkv = wide[:, :width]
    cache, batch = A.KVCache(c.k, c.v), c.batch(A)
    q = torch.empty(tokens, hq, d, dtype=c.T, device="cuda")
    w, cpos = cache.weights() + 1.0, torch.full((4, 41), -7, dtype=torch.int32, device="cuda")
    before_k, before_v = c.k.float().cpu().numpy(), c.v.float().cpu().numpy()
    rope = A.Rope(cos, sin, sections, interleaved)
    A.rope_append(cache, batch, rope, qkv, torch.from_numpy(pos).cuda(), q, w, cpos)
    h = qkv.float().cpu().numpy().reshape(tokens, hq + 2 * hkv, d)
    want = orc.rotate(h[:, :hq + hkv], cos.cpu().numpy(), sin.cpu().numpy(), pos, sections, interleaved)
    big = np.abs(h[:, :hq + hkv]).max(-1, keepdims=True)   # two products and a sum in fp32, then the rounding to the type
    bound = lambda y: 4 * U * 2 * big[:, :1].max() + (2.0 ** -8 if dtype == "bf16" else 0) * np.abs(y)  # noqa: E731
    assert np.all(np.abs(q.float().cpu().numpy() - want[:, :hq]) <= bound(want[:, :hq]))
    k, v, row = c.k.float().cpu().numpy(), c.v.float().cpu().numpy(), 0
    touched = np.zeros(tuple(c.k.shape[:3]), bool)
    want_pos = np.full((4, 41), -7)
    for b, (n, new) in enumerate(zip(lens, news)):
        for t in range(new):
            j = n - new + t
            p, s = c.table_np[b, j // page], j % page
            touched[p, :, s] = True
            want_pos[b, j] = pos[0, row]
            y = want[row, hq:]
            assert np.all(np.abs(k[p, :, s] - y) <= bound(y))
            vv = h[row, hq + hkv:]
            assert np.all(np.abs(v[p, :, s] - vv) <= (2.0 ** -8 * np.abs(vv) if dtype == "bf16" else 0))
            row += 1
    assert np.array_equal(k[~touched], before_k[~touched], equal_nan=True) and np.array_equal(v[~touched], before_v[~touched], equal_nan=True)
    assert np.array_equal(w.cpu().numpy(), np.where(touched, 0.0, 1.0)) and np.array_equal(cpos.cpu().numpy(), want_pos)


def test_rope_append_one_token_each_and_pages_that_do_not_exist(A):
    import torch
    c = Case("bf16", 64, 4, 2, 16, [33, 16, 0], [1, 1, 1], gone={(0, 2)}, one_new=True)
    angle = np.linspace(0, 1, 50)[:, None] * np.ones((1, 32))
    rope = A.Rope(torch.from_numpy(np.cos(angle).astype(np.float32)).cuda(), torch.from_numpy(np.sin(angle).astype(np.float32)).cuda())
    qkv = torch.ones(3, 8 * 64, device="cuda")
    q = torch.full((3, 4, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    before = c.k.clone()
    pos = torch.tensor([[49, -3, 1000]], dtype=torch.int32).cuda()            # positions are cut to the tables' rows
    A.rope_append(A.KVCache(c.k, c.v), c.batch(A), rope, qkv, pos, q)
    same = torch.isclose(c.k.float(), before.float(), equal_nan=True)
    assert int((~same).any(-1).sum()) == 2                                      # sequence 1's token, both heads
    assert torch.isfinite(q.float()).all() and torch.equal(q[0], q[2]) and (q[1] == 1).all()


# ---------------------------------------------------------------- eviction
@pytest.mark.parametrize("dtype,d,hkv,page", [("bf16", 64, 2, 16), ("f32", 40, 3, 8), ("bf16", 128, 1, 64), ("bf16", 8, 5, 16)])
@pytest.mark.parametrize("keep,sinks,recent", [(50, 4, 10), (1, 0, 0), (64, 0, 64), (500, 3, 3), (0, 0, 0), (97, 97, 0)])
def test_eviction(A, dtype, d, hkv, page, keep, sinks, recent):
    import torch
    rng = np.random.default_rng(keep)
    lens = [1100, 64, 0, 1, 97, 300]
    c = Case(dtype, d, hkv, hkv, page, lens, [1] * 6, gone={(0, 2), (4, 0)}, spare=6 * (500 // page + 2))
    w = torch.from_numpy(np.floor(rng.exponential(1.0, tuple(c.k.shape[:3])) * 4).astype(np.float32) / 4)   # many equal ones
    w[c.table_np[5, 1], 0, 3], w[c.table_np[5, 0], 0, 1], w[c.table_np[5, 1], 0, 2] = float("nan"), float("inf"), -1.0
    w = w.cuda()
    named = set(c.table_np.flatten().tolist())
    free = [p for p in rng.permutation(c.pages) if p not in named]
    per = max(1, -(-keep // page))
    out = np.array(free[:6 * per], np.int32).reshape(6, per)
    pos = rng.integers(0, 1 << 30, (6, 1200)).astype(np.int32)
    cache, batch = A.KVCache(c.k, c.v), A.Batch(c.table, c.length, max_len=1100)
    full = lambda *s: torch.full(s, -9, dtype=torch.int32, device="cuda")  # noqa: E731
    length, kept, pos_out = full(6), full(6, keep), full(6, keep)
    ws = torch.full((A.cache_evict_workspace_size(cache, batch),), 0xff, dtype=torch.uint8, device="cuda")
    k0, v0, w0 = (x.float().cpu().numpy() for x in (c.k, c.v, w))
    A.cache_evict(cache, batch, c.i32(out), w, keep, sinks, recent, length, kept, torch.from_numpy(pos).cuda(), pos_out, ws)
    k1, v1, w1, kept, pos_out = (x.float().cpu().numpy() if x.dtype != torch.int32 else x.cpu().numpy() for x in (c.k, c.v, w, kept, pos_out))
    for b, n in enumerate(lens):
        at = [(c.table_np[b, j // page], j % page) for j in range(n)]
        mine = np.array([w0[p, :, s] if c.exists[b][j] else np.zeros(hkv) for j, (p, s) in enumerate(at)], np.float32).reshape(n, hkv)
        want = orc.kept(mine, keep, sinks, recent, c.exists[b])
        assert int(length[b]) == len(want)
        assert kept[b, :len(want)].tolist() == want.tolist() and (kept[b, len(want):] == -1).all()
        assert pos_out[b, :len(want)].tolist() == pos[b, want].tolist() and (pos_out[b, len(want):] == -1).all()
        for i, j in enumerate(want):
            p, s = at[j]
            for new, old in ((k1, k0), (v1, v0), (w1, w0)):
                assert np.array_equal(new[out[b, i // page], :, i % page], old[p, :, s], equal_nan=True)
    stay = np.setdiff1d(np.arange(c.pages), out.flatten())
    assert np.array_equal(k1[stay], k0[stay], equal_nan=True) and np.array_equal(w1[stay], w0[stay], equal_nan=True)


def test_refusals_come_as_errors(A):
    import torch
    from paper_2605_00422_amd import binding as B
    c = Case("bf16", 64, 4, 2, 16, [900], [1], one_new=True)
    cache, batch, q = A.KVCache(c.k, c.v), c.batch(A), c.q.cuda()
    with pytest.raises(B.BwlaError):
        A.attention_forward(cache, batch, A.Score(-0.1), q, torch.empty_like(q))
    with pytest.raises(B.BwlaError):
        A.attention_forward(cache, batch, A.Score(0.1), q, torch.empty_like(q), None, cache.weights())
    with pytest.raises(B.BwlaError):
        A.attention_forward(cache, batch, A.Score(0.1), q, torch.empty_like(q), None, None, None)


# ---------------------------------------------------------------- all of it, between two layers
def test_attention_block_against_the_oracle_step_by_step(A):
    """A prompt, its cache cut, a decoding step: each operator's outputs against the oracle's on what it read (bf16, all of a
    kernel's bounds as above); the layers on either side are other tests' matter."""
    import torch
    from paper_2605_00422_amd import attention_block as T
    hq, hkv, d, page, hidden, m, keep = 4, 2, 64, 16, 512, 200, 40
    gen = torch.Generator(device="cuda").manual_seed(3)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    k, v = (torch.full((20, hkv, page, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rope = T.tables(torch, m + 8, d, "cuda")
    block = T.AttentionBlock(T.random_layer(torch, gen, (hq + 2 * hkv) * d, hidden, 8, "cuda"),
                             T.random_layer(torch, gen, hidden, hq * d, 8, "cuda"), A.KVCache(k, v), rope, hq)
    table, length = i32([list(range(13))]), i32([m])
    cos, sin = rope.cos.cpu().numpy(), rope.sin.cpu().numpy()

    def cached(pages, n):
        return (np.concatenate([x[p].float().cpu().numpy().transpose(1, 0, 2) for p in pages])[:n] for x in (k, v))

    def check_call(rows, pages, n, position):
        _, qkv, q, out, lse, _ = block._rows[rows]
        heads = qkv.cpu().numpy().astype(np.float64).reshape(rows, hq + 2 * hkv, d)
        turned = orc.rotate(heads[:, :hq + hkv], cos, sin, [position], [d // 2])
        kb, vb = cached(pages, n)
        most = np.abs(heads).max()
        for got, want in ((q.float().cpu().numpy(), turned[:, :hq]), (kb[n - rows:], turned[:, hq:]), (vb[n - rows:], heads[:, hq + hkv:])):
            assert np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 8 * U * most)
        want, want_lse, sums, vabs, qk, top = orc.attend(q.float().cpu().numpy(), kb, vb, d ** -0.5)
        rel = np.expm1(4 * (d + 4) * U * qk + 16 * U * top) + (2 * n + 16) * U
        assert np.all(np.abs(out.float().cpu().numpy() - want) <= vabs * (rel[..., None] + 2.0 ** -9) + np.abs(want) * 2.0 ** -8 + 1e-30)
        assert np.all(np.abs(lse.cpu().numpy() - want_lse) <= rel + 8 * U * (np.abs(want_lse) + 1))
        return sums, (rel + 8 * U * (np.abs(want_lse) + top)).max() + (rows * 2 + 8) * U

    x, y = torch.randn(m, hidden, generator=gen, device="cuda").bfloat16(), torch.empty(m, hidden, device="cuda")
    batch = A.Batch(table, length, i32([0, m]), tokens=m, max_new=m, max_len=m)
    block(x, batch, i32([list(range(m))]), y)
    want, bound = check_call(m, range(13), m, list(range(m)))
    sums = np.concatenate([block.sums[p].cpu().numpy().T for p in range(13)])[:m]
    assert np.all(np.abs(sums - want) <= want * bound)
    assert torch.isfinite(y).all()
    _, _, _, out, _, act = block._rows[m]
    again = torch.empty_like(y)                        # the output layer read what the attention wrote
    from paper_2605_00422_amd import binding as B
    assert torch.equal(y, B.decode_forward(block.o, out.view(m, -1), act, again))
    stay = orc.kept(sums, keep, 4, 8)
    k0, v0 = cached(range(13), m)
    table_out, left = i32([[13, 14, 15, 16]]), i32([0])
    block.cut(batch, table_out, keep, 4, 8, left)
    k1, v1 = cached(range(13, 17), keep)
    assert int(left) == keep and np.array_equal(k1, k0[stay]) and np.array_equal(v1, v0[stay])
    left += 1
    x, y = torch.randn(1, hidden, generator=gen, device="cuda").bfloat16(), torch.empty(1, hidden, device="cuda")
    block(x, A.Batch(table_out, left, max_len=keep + 1), i32([[m]]), y)
    check_call(1, range(13, 17), keep + 1, [m])
    assert torch.isfinite(y).all()


def test_attention_block_example(A):
    import torch
    from paper_2605_00422_amd import attention_block as T
    ys, lens = T.main()
    assert [tuple(y.shape) for y in ys] == [(300, 512), (77, 512)] + [(2, 512)] * 16 and all(torch.isfinite(y).all() for y in ys)
    assert lens.tolist() == [[64 + i, 64 + i] for i in range(1, 17)]
    again, _ = T.main()
    assert all(torch.equal(a, b) for a, b in zip(ys, again))
