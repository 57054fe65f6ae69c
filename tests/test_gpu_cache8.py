"""Norms of heads in the rotation's pass, and the cache of 8-bit codes that it writes, against the fp64 oracle.

Bounds, derived from the arithmetic (u = 2^-24).  Norm: the sum of d squares is off by d u of itself at most, its root by half of that,
and the division, root (2 u), mean and two products add about 8 u: (d / 2 + 8) u |y|; centered, the mean adds (d + 2) u mean|x| to each
x - mu.  Rotation: two products and a sum, 2 u (|a cos| + |b sin|) and what their factors bring.  Together E, a bound of what a value
is off before it is stored.  bf16: 2^-8 of the value more.  Codes: the scale is off by E / top + 2 u of itself (and so by the doubling next
to it where the values lie within that of a border, which the cases' seeds do not); a value is off by half a step (of its code),
where code numbers are off by E / scale and 4 u of themselves: a code may fall to the neighbour where it lies that near to a middle, so that
value and oracle differ by a step there, and by the scale's error times the code everywhere.
"""
import numpy as np
import pytest

from oracle import bwla_attention_oracle as att
from oracle import bwla_cache8_oracle as orc

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def A():
    pytest.importorskip("torch")                       # (in front of the library: one HIP runtime for both)
    from paper_2605_00422_amd import attention_binding
    attention_binding.load()
    return attention_binding


class Call:
    """Rows of a merged projection, sequences of lens cached tokens of which the last news are new, a norm and a rotation."""

    def __init__(self, A, hq=4, hkv=2, d=64, page=16, lens=(20, 3, 40), news=(1, 3, 25), pairs=None, axes=1, interleaved=False, norm="rms",
                 x="f32", dtype="bf16", seed=0, one_new=False, spread=1.0):
        import torch
        self.torch, self.A, self.hq, self.hkv, self.d, self.page, self.lens, self.news = torch, A, hq, hkv, d, page, list(lens), list(news)
        rng = self.rng = np.random.default_rng(seed)
        self.types = {"bf16": torch.bfloat16, "f32": torch.float32}
        self.dtype, self.T = dtype, self.types[dtype]
        n, self.tokens = len(lens), sum(news)
        per = max(1, max(-(-x // page) for x in lens))
        self.pages = n * per + 2
        self.table_np = rng.permutation(self.pages)[:n * per].reshape(n, per).astype(np.int32)
        i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32).cuda()  # noqa: E731
        self.i32, self.table, self.length = i32, i32(self.table_np), i32(lens)
        self.first = None if one_new else i32(np.concatenate([[0], np.cumsum(news)]))
        qkv = rng.standard_normal((self.tokens, (hq + 2 * hkv) * d)) * spread
        self.qkv = torch.from_numpy(qkv.astype(np.float32)).to(self.types[x])
        pairs = d // 2 if pairs is None else pairs
        self.sections = [pairs] if axes == 1 else [pairs // 3] * (axes - 1) + [pairs - pairs // 3 * (axes - 1)]
        rows = 50
        angle = np.arange(rows)[:, None] * 100.0 ** (-np.arange(pairs) / max(pairs, 1))
        self.cos, self.sin = np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)
        self.pos = rng.integers(0, rows, (axes, self.tokens)).astype(np.int32)
        self.interleaved, self.kind = interleaved, norm
        w = lambda h: rng.uniform(0.5, 1.5, (h, d) if norm == "heads" else (d,)).astype(np.float32)  # noqa: E731
        self.wq, self.wk = (w(hq), w(hkv)) if norm not in ("none", "bare") else (None, None)
        up = lambda v: None if v is None else torch.from_numpy(v).cuda()  # noqa: E731
        self.norm = None if norm == "none" else A.HeadNorm(up(self.wq), up(self.wk), 1e-5, centered=norm == "centered")
        self.rope = A.Rope(up(self.cos), up(self.sin), self.sections, interleaved)
        self.q = torch.full((self.tokens, hq, d), 9.0, dtype=self.T, device="cuda")

    def batch(self, **kw):
        d = dict(tokens=self.tokens, max_new=max(self.news), max_len=max(self.lens))
        return self.A.Batch(self.table, self.length, self.first, **{**d, **kw})

    def append(self, cache, **kw):
        self.A.norm_rope_append(cache, kw.pop("batch", None) or self.batch(), self.rope, self.norm, self.qkv.cuda(), self.i32(self.pos), self.q, **kw)

    def want(self):
        """(queries, keys, values) of each row, and bounds of their errors in fp32."""
        x = self.qkv.double().numpy().reshape(self.tokens, -1, self.d)
        parts, off = [], []
        for lo, n, w in ((0, self.hq, self.wq), (self.hq, self.hkv, self.wk)):
            y = x[:, lo:lo + n]
            e = np.zeros_like(y)
            if self.kind != "none":
                raw, y = y, orc.norm(y, w, 1e-5, self.kind == "centered")
                e = (self.d / 2 + 10) * U * np.abs(y)
                if self.kind == "centered":
                    rms = np.sqrt(((raw - raw.mean(-1, keepdims=True)) ** 2).mean(-1, keepdims=True) + 1e-5)
                    wide = (self.d + 2) * U * np.abs(raw).mean(-1, keepdims=True) / rms
                    e = e + wide * (1.5 + np.abs(y))
            parts.append(att.rotate(y, self.cos, self.sin, self.pos, self.sections, self.interleaved))
            # (an angle mixes a pair's errors: no more than both together)
            off.append(2 * e.max(-1, keepdims=True) + 4 * U * np.abs(y).max(-1, keepdims=True) + np.zeros_like(y))
        parts.append(x[:, self.hq + self.hkv:])
        off.append(np.zeros_like(parts[2]))
        return parts, off

    def rows_of(self):
        """(sequence, first index, rows) of each sequence's new tokens."""
        row = 0
        for b, (n, m) in enumerate(zip(self.lens, self.news)):
            yield b, n - m, range(row, row + m)
            row += m


def store_bound(dtype, y):
    return np.abs(y) * (2.0 ** -8 if dtype == "bf16" else U) + 1e-38


SHAPES = [dict(), dict(d=128, hq=5, hkv=1), dict(d=96, pairs=24), dict(d=80, pairs=20, axes=2), dict(d=256, axes=3), dict(d=16, pairs=3), dict(d=256, pairs=5),
          dict(d=64, pairs=0), dict(d=112, pairs=56, interleaved=True), dict(d=64, pairs=12, interleaved=True, axes=4), dict(d=240, pairs=8), dict(hq=33, hkv=3)]


@pytest.mark.parametrize("norm", ["rms", "heads", "centered", "bare", "none"])
@pytest.mark.parametrize("shape", SHAPES)
def test_normed_and_turned(A, shape, norm):
    import torch
    for x, dtype in (("f32", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("bf16", "bf16")):
        c = Call(A, norm=norm, x=x, dtype=dtype, seed=4, **shape)
        k, v = (torch.full((c.pages, c.hkv, c.page, c.d), 9.0, dtype=c.T, device="cuda") for _ in range(2))
        cache = A.KVCache(k, v)
        sums = cache.weights() + 3
        cpos = torch.full((3, 40), 77, dtype=torch.int32, device="cuda")
        c.append(cache, weights=sums, cache_position=cpos)
        (q, kk, vv), (eq, ek, _) = c.want()
        assert np.all(np.abs(c.q.double().cpu().numpy() - q) <= eq + store_bound(dtype, np.abs(q) + eq))
        untouched = np.ones((c.pages, c.page), bool)
        for b, j, rows in c.rows_of():
            for i, r in enumerate(rows):
                p, s = c.table_np[b, (j + i) // c.page], (j + i) % c.page
                untouched[p, s] = False
                assert np.all(np.abs(k[p, :, s].double().cpu().numpy() - kk[r]) <= ek[r] + store_bound(dtype, np.abs(kk[r]) + ek[r]))
                assert np.all(np.abs(v[p, :, s].double().cpu().numpy() - vv[r]) <= store_bound(dtype, vv[r]))
                assert int(cpos[b, j + i]) == c.pos[0, r] and not sums[p, :, s].any()
        keep = torch.from_numpy(untouched).cuda()
        assert (k.transpose(1, 2)[keep] == 9).all() and (v.transpose(1, 2)[keep] == 9).all() and (sums.transpose(1, 2)[keep] == 3).all()


def test_without_a_norm_it_is_rope_append(A):
    import torch
    c = Call(A, norm="none", d=128)
    outs = []
    for call in (lambda cache: c.append(cache), lambda cache: A.rope_append(cache, c.batch(), c.rope, c.qkv.cuda(), c.i32(c.pos), c.q)):
        k, v = (torch.zeros(c.pages, c.hkv, c.page, c.d, dtype=c.T, device="cuda") for _ in range(2))
        call(A.KVCache(k, v))
        outs.append((k, v, c.q.clone()))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.parametrize("size", [1e-25, 1e-12, 1e18, 3e19, 1e30, 3e37])
def test_norms_of_very_small_and_very_large_heads(A, size):
    """Squares below and beyond fp32's range."""
    import torch
    c = Call(A, spread=1.0, dtype="f32", d=128, norm="rms")
    c.qkv = (c.qkv.double() * size).float()
    k, v = (torch.zeros(c.pages, c.hkv, c.page, c.d, device="cuda") for _ in range(2))
    c.append(A.KVCache(k, v))
    (q, _, _), (eq, _, _) = c.want()
    got = c.q.double().cpu().numpy()
    assert np.isfinite(got).all() and np.all(np.abs(got - q) <= eq + store_bound("f32", q))


# ---------------------------------------------------------------- codes
def make8(c, code, fill=None, strided=False):
    import torch
    T = torch.int8 if code == "i8" else torch.float8_e4m3fn
    shape = (c.pages, c.hkv, c.page, c.d)
    if fill is not None:
        raw = np.full(shape, fill, np.uint8)
    elif code == "i8":
        raw = c.rng.integers(-127, 128, shape).astype(np.int8).view(np.uint8)
    else:
        raw = (c.rng.integers(0, 127, shape) + 128 * c.rng.integers(0, 2, shape)).astype(np.uint8)
    raw = torch.from_numpy(raw).cuda()
    k, v = raw.clone(), raw.flip(0).clone()
    if strided:                                        # (page, slot, head, column) in memory, rows 32 bytes apart
        wide = torch.zeros(2, c.pages, c.page, c.hkv, c.d + 32, dtype=torch.uint8, device="cuda")
        wide[0, ..., :c.d], wide[1, ..., :c.d] = k.transpose(1, 2), v.transpose(1, 2)
        k, v = (wide[i, ..., :c.d].transpose(1, 2) for i in range(2))
    ks, vs = (torch.from_numpy(c.rng.uniform(0.001, 0.02, (c.pages, c.hkv + 1)).astype(np.float32)).cuda()[:, :c.hkv] for _ in range(2))
    return c.A.KVCache8(k.view(T), v.view(T), ks, vs, c.T)


def numbers(t):
    return t.double().cpu().numpy()


def check8(A, c, code, cache, **kw):
    """The append against the oracle, page by page; what lies elsewhere stays to the bit."""
    import torch
    before = [(numbers(t), numbers(s)) for t, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale))]
    raw = [t.view(torch.uint8).clone() for t in (cache.k, cache.v)]
    c.append(cache, **kw)
    parts, off = c.want()
    assert np.all(np.abs(numbers(c.q) - parts[0]) <= off[0] + store_bound(c.dtype, np.abs(parts[0]) + off[0]))
    touched = np.zeros((c.pages, c.page), bool)
    flips = total = 0
    for which, (t, scale, y, e) in enumerate(((cache.k, cache.k_scale, parts[1], off[1]), (cache.v, cache.v_scale, parts[2], off[2]))):
        got, got_scale = numbers(t), numbers(scale)
        codes, scales = before[which]
        codes = np.nan_to_num(codes, nan=0.0)
        for b, j, rows in c.rows_of():
            j0, at = j, 0
            while at < len(rows):
                up = min(len(rows), at + c.page - j0 % c.page)
                p, inside = c.table_np[b, j0 // c.page], j0 % c.page
                touched[p, :inside + up - at] = True
                for h in range(c.hkv):
                    mine = y[rows[at]:rows[up - 1] + 1, h]
                    old = codes[p, h].copy()
                    want_scale, doubled = orc.append(code, old, scales[p, h], mine, inside)
                    tol = e[rows[at]:rows[up - 1] + 1, h].max() / orc.TOP[code] + 3 * U * want_scale + 1e-44
                    assert abs(got_scale[p, h] - want_scale) <= tol, (b, p, h, got_scale[p, h], want_scale)
                    # older codes: exactly those of the oracle
                    assert np.array_equal(got[p, h, :inside], old[:inside]), (b, p, h)
                    new, want = got[p, h, inside:inside + up - at], old[inside:inside + up - at]
                    if want_scale > 0:
                        number = np.nan_to_num(mine / want_scale, nan=0.0, posinf=1e30, neginf=-1e30)
                        number = np.clip(number, -orc.TOP[code], orc.TOP[code])
                        step = orc.step_of(code, number)
                        near = e[rows[at]:rows[up - 1] + 1, h] / want_scale * 2 + 8 * U * np.abs(number)
                        differs = new != want
                        # another code: its neighbour, where the number lies in the middle but for its error
                        middle = np.abs(np.abs(number / step - np.floor(number / step)) - 0.5) * step
                        assert np.all(~differs | ((np.abs(new - want) <= step * 1.001) & (middle <= near + 1e-30))), (b, p, h)
                        flips += int(differs.sum())
                        total += differs.size
                    else:
                        assert not new.any()
                j0 += up - at
                at = up
    for t, r, scale, (_, s0) in zip((cache.k, cache.v), raw, (cache.k_scale, cache.v_scale), before):
        keep = torch.from_numpy(~touched).cuda()
        assert torch.equal(t.view(torch.uint8).transpose(1, 2)[keep], r.transpose(1, 2)[keep])
        none = ~touched.any(1)
        assert np.array_equal(numbers(scale)[none], s0[none])
    # (Of fp32 values hardly any lie that near to a middle.  Of bf16 ones, of 8 bits, up to one in 2^4 lies on a middle of e4m3 codes, of 4 bits,
    # where a page's largest is 1.75 times a power of two, so that its scale is one: rounded to fp32 that is exact, and value / scale a tie; in
    # other pages the oracle's scale, which is not rounded, moves such numbers off the middle by up to u of themselves.)
    assert flips <= 3 + (total / 16 if c.qkv.dtype is not torch.float32 else total * 1e-3)
    return cache


CODES = ["i8", "e4m3"]


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("shape", SHAPES)
def test_codes_of_every_shape(A, code, shape):
    for x, dtype in (("f32", "bf16"), ("bf16", "f32")):
        c = Call(A, x=x, dtype=dtype, seed=6, **shape)
        check8(A, c, code, make8(c, code))


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("norm", ["heads", "centered", "bare", "none"])
def test_codes_with_every_norm(A, code, norm):
    c = Call(A, norm=norm, d=128, hq=8, lens=(100, 16, 33, 1), news=(1, 16, 18, 1), seed=3)
    check8(A, c, code, make8(c, code))


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("page,lens,news", [
    (8, (7, 8, 9, 1, 16), (1, 1, 1, 1, 1)), (8, (20, 33), (20, 27)), (16, (64, 17), (64, 17)), (64, (200, 70, 65), (130, 3, 65)),
    (128, (300, 129), (290, 2)), (512, (700, 30), (690, 30)), (2048, (1500,), (1400,)), (16, (5, 0, 30), (0, 0, 14))])
def test_codes_of_pages_and_lengths(A, code, page, lens, news):
    c = Call(A, page=page, lens=lens, news=news, seed=7, one_new=set(news) == {1})
    check8(A, c, code, make8(c, code))
    c = Call(A, page=page, lens=lens, news=news, seed=8, d=16, pairs=3)
    check8(A, c, code, make8(c, code, strided=True))


@pytest.mark.parametrize("code", CODES)
def test_scales_grow_and_older_codes_follow(A, code):
    """Tokens one by one, each larger than the one before by up to 2^7."""
    c = Call(A, lens=(1, 9, 30), news=(1, 1, 1), one_new=True, norm="none", seed=9)
    cache = make8(c, code)
    for step in range(1, 9):
        c.qkv = (c.qkv.float() * c.rng.choice([0.5, 1.0, 3.0, 128.0])).clamp(-1e30, 1e30)
        check8(A, c, code, cache)
        c.lens = [n + 1 if (n + 1) % 16 else n for n in c.lens]
        c.length = c.i32(c.lens)
        if max(c.lens) > 16 * c.table_np.shape[1]:
            break


@pytest.mark.parametrize("code", CODES)
def test_zeros_scales_of_zero_and_values_that_are_not_finite(A, code):
    import torch
    c = Call(A, norm="none", lens=(20, 18, 40, 7), news=(3, 18, 4, 1), seed=10)
    cache = make8(c, code)
    first = np.concatenate([[0], np.cumsum(c.news)])
    c.qkv[first[0]:first[1], c.hq * c.d:] = 0                                    # nothing but zeros behind older tokens
    c.qkv[first[1]:first[2], c.hq * c.d:] = 0                                    # ... in fresh pages: scales of 0
    c.qkv[first[2] + 1, c.hq * c.d + 5] = float("nan")
    c.qkv[first[2] + 2, (c.hq + c.hkv) * c.d + 7] = float("inf")
    c.qkv[first[2], (c.hq + c.hkv) * c.d + 9] = -float("inf")
    cache.k_scale[int(c.table_np[3, 0])] = 0                                     # older tokens, but no scale yet
    (q, k, v), off = c.want()
    ok = np.isfinite(k).all(-1)
    c.append(cache)
    for b, j, rows in c.rows_of():
        for i, r in enumerate(rows):
            p, s = c.table_np[b, (j + i) // 16], (j + i) % 16
            for h in range(c.hkv):
                for t, scale, y, e in ((cache.k, cache.k_scale, k, off[1]), (cache.v, cache.v_scale, v, off[2])):
                    got, sc = numbers(t[p, h, s]), float(scale[p, h])
                    assert np.isfinite(sc) and np.isfinite(got).all()
                    fin = np.isfinite(y[r, h])
                    with np.errstate(invalid="ignore"):
                        assert np.all((np.abs(got * sc - y[r, h]) <= 0.51 * sc * orc.step_of(code, got) + np.nan_to_num(e[r, h], nan=1e-3))[fin])
                    assert np.all(got[np.isposinf(y[r, h])] == orc.TOP[code]) and np.all(got[np.isneginf(y[r, h])] == -orc.TOP[code])
                    assert not got[np.isnan(y[r, h])].any()
    assert ok.any()
    assert not cache.k_scale[int(c.table_np[1, 0])].any() and not numbers(cache.k[int(c.table_np[1, 0])]).any()
    assert float(cache.k_scale[int(c.table_np[3, 0])].min()) > 0


@pytest.mark.parametrize("code", CODES)
def test_pages_of_zeros_and_infinities_have_codes_of_zero(A, code):
    """Nothing finite but zeros: the scale is 0, and so is every code."""
    c = Call(A, norm="none", lens=(20,), news=(18,), seed=10)
    cache = make8(c, code)
    c.qkv[:, c.hq * c.d:] = 0
    c.qkv[3, (c.hq + c.hkv) * c.d + 7] = float("inf")
    c.qkv[4, (c.hq + c.hkv) * c.d + 8] = -float("inf")
    c.append(cache)
    p, s = c.table_np[0, 5 // 16], 5 % 16              # (rows 3 and 4 are tokens 5 and 6: of a page with older tokens)
    assert float(cache.v_scale[int(p)].min()) > 0
    assert numbers(cache.v[int(p), 0, s])[7] == orc.TOP[code] and numbers(cache.v[int(p), 0, s + 1])[8] == -orc.TOP[code]
    fresh = Call(A, norm="none", lens=(18,), news=(18,), seed=11)
    cache = make8(fresh, code)
    fresh.qkv[:, fresh.hq * fresh.d:] = 0
    fresh.qkv[3, (fresh.hq + fresh.hkv) * fresh.d + 7] = float("inf")
    fresh.qkv[4, (fresh.hq + fresh.hkv) * fresh.d + 8] = -float("inf")
    fresh.append(cache)
    p = int(fresh.table_np[0, 0])
    assert not cache.v_scale[p].any() and not numbers(cache.v[p, :, :16]).any()


@pytest.mark.parametrize("code", CODES)
def test_sequences_without_new_tokens_stay_as_they_were(A, code):
    import torch
    c = Call(A, lens=(20, 37, 5), news=(2, 0, 0), seed=21)
    cache = make8(c, code)
    for p in c.table_np[1:].ravel():
        cache.k_scale[int(p)] = -3.0                   # (no scale; a call that has nothing to write there leaves it)
        cache.v_scale[int(p)] = float("nan")
    before = [t.view(torch.uint8).clone() for t in (cache.k, cache.v)] + [cache.k_scale.view(torch.int32).clone(), cache.v_scale.view(torch.int32).clone()]
    c.append(cache)
    after = [t.view(torch.uint8) for t in (cache.k, cache.v)] + [cache.k_scale.view(torch.int32), cache.v_scale.view(torch.int32)]
    for x, y in zip(before, after):
        for p in c.table_np[1:].ravel():
            assert torch.equal(x[int(p)], y[int(p)])


@pytest.mark.parametrize("code", CODES)
def test_rows_and_pages_that_are_left_out(A, code):
    """Rows of no sequence, more new tokens than max_new, new tokens in front of the cache, pages that do not exist: nothing is written."""
    import torch
    c = Call(A, lens=(40, 5, 30), news=(10, 9, 30), seed=11)
    cache = make8(c, code)
    c.table_np[2, 1] = -1
    c.table = c.i32(c.table_np)
    first = c.i32([2, 12, 21, 51])
    c.tokens += 4
    c.qkv = torch.cat([c.qkv[:2], c.qkv, c.qkv[:2]])
    c.pos = np.concatenate([c.pos[:, :2], c.pos, c.pos[:, :2]], 1)
    c.q = torch.full((c.tokens, c.hq, c.d), 9.0, dtype=c.T, device="cuda")
    k0, s0 = cache.k.view(torch.uint8).clone(), cache.k_scale.clone()
    c.append(cache, batch=A.Batch(c.table, c.length, first, tokens=c.tokens, max_new=20, max_len=40))
    changed = (cache.k.view(torch.uint8) != k0).transpose(1, 2).flatten(2).any(2).cpu().numpy()
    allowed = np.zeros_like(changed)
    allowed[c.table_np[0, 1], 14:] = allowed[c.table_np[0, 2], :8] = True        # tokens 30 .. 39, and older codes that follow
    allowed[c.table_np[0, 1], :14] = True
    allowed[c.table_np[1, 0], :5] = True                                         # 9 new ones of 5: the last five
    allowed[c.table_np[2, 0]] = True                                             # the first 20 of 30, of which 4 have no page
    assert not (changed & ~allowed).any() and changed[c.table_np[2, 0]].any()
    assert (c.q[:2] == 9).all() and (c.q[51:] == 9).all() and (c.q[2 + 19 + 20:51] == 9).all() and not (c.q[2:41] == 9).all(-1).any()
    used = [c.table_np[0, 1], c.table_np[0, 2], c.table_np[1, 0], c.table_np[2, 0]]
    others = np.setdiff1d(np.arange(c.pages), used)
    assert torch.equal(cache.k_scale[others], s0[others])


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_values_read_back(A, code, out):
    import torch
    c = Call(A, lens=(40, 0, 17), news=(1, 0, 1), d=48, pairs=8, seed=12)
    cache = make8(c, code, fill=0x31)
    c.table_np[0, 1] = c.pages + 4
    T = c.types[out]
    batch = A.Batch(c.i32(c.table_np), c.length, max_len=40)
    k, v = (torch.full((3, 40, c.hkv, c.d), 9.0, dtype=T, device="cuda") for _ in range(2))
    A.cache8_read(cache, batch, k, v)
    only = torch.full_like(v, 9.0)
    A.cache8_read(cache, batch, v=only)
    assert torch.equal(only, v)
    for t, codes, scale in ((k, cache.k, cache.k_scale), (v, cache.v, cache.v_scale)):
        want = torch.zeros(3, 40, c.hkv, c.d, dtype=torch.float32, device="cuda")
        for b in range(3):
            for j in range(c.lens[b]):
                p = int(c.table_np[b, j // 16])
                if p < c.pages:
                    want[b, j] = codes[p, :, j % 16].float() * scale[p][:, None]  # one product of fp32, rounded once more to the output's type
        assert torch.equal(t, want.to(T))


@pytest.mark.parametrize("code", CODES)
def test_pages_beyond_32_bits(A, code):
    import torch
    T = torch.int8 if code == "i8" else torch.float8_e4m3fn
    pages = (1 << 32) // (8 * 64 * 128) + 40
    c = Call(A, hq=8, hkv=8, d=128, page=64, lens=(130, 70), news=(70, 1), seed=13)
    k = torch.zeros(pages, 8, 64, 128, dtype=torch.uint8, device="cuda")
    v, ks, vs = torch.zeros_like(k), torch.ones(pages, 8, device="cuda"), torch.ones(pages, 8, device="cuda")
    small = make8(c, code, fill=1)
    small.k_scale.fill_(1), small.v_scale.fill_(1)
    k[pages - 40:], v[pages - 40:] = 1, 1
    far = pages - 1 - c.table_np
    for cache, table in ((small, c.table_np), (A.KVCache8(k.view(T), v.view(T), ks, vs, c.T), far)):
        c.append(cache, batch=A.Batch(c.i32(table), c.length, c.first, tokens=c.tokens, max_new=70, max_len=130))
    for p, f in zip(c.table_np.flatten(), far.flatten()):
        assert torch.equal(small.k.view(torch.uint8)[p], k[f]) and torch.equal(small.v.view(torch.uint8)[p], v[f])
        assert torch.equal(small.k_scale[p], ks[f]) and torch.equal(small.v_scale[p], vs[f])


def test_one_token_at_a_time_ends_where_the_bound_says(A):
    """A cache written token by token and one written at once stand for the same values, but for a step of the last scale."""
    import torch
    c = Call(A, lens=(37,), news=(37,), norm="rms", d=64, seed=14)
    whole, steps = make8(c, "i8", fill=0), make8(c, "i8", fill=0)
    c.append(whole)
    rows, pos = c.qkv.clone(), c.pos
    for j in range(37):
        length = c.i32([j + 1])
        q = torch.empty(1, c.hq, c.d, dtype=c.T, device="cuda")
        A.norm_rope_append(steps, A.Batch(c.table, length, max_len=37), c.rope, c.norm, rows[j:j + 1].cuda(), c.i32(pos[:, j:j + 1]), q)
    out = [torch.empty(1, 37, c.hkv, c.d, device="cuda") for _ in range(4)]
    batch = A.Batch(c.table, c.i32([37]), max_len=37)
    A.cache8_read(whole, batch, *out[:2])
    A.cache8_read(steps, batch, *out[2:])
    scale = steps.k_scale[c.table.long()][0].repeat_interleave(16, 0)[:37, :, None], steps.v_scale[c.table.long()][0].repeat_interleave(16, 0)[:37, :, None]
    for a, b, s in zip(out[:2], out[2:], scale):
        assert ((a - b).abs() <= 1.51 * s).all()       # (half a step of the other's smaller scale besides)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("old", [0.0, 1e-44, 1e-39, 2.0 ** -126])
def test_scales_of_older_tokens_at_the_edge_of_fp32(A, code, old):
    """A scale of 0 makes zeros of older codes; one without a reciprocal in fp32 is doubled until it has one, whatever the new values."""
    for size in (1.0, 1e-37, 1e-41):
        c = Call(A, norm="none", lens=(20, 33), news=(2, 1), seed=15, spread=size)
        cache = make8(c, code)
        cache.k_scale.fill_(old), cache.v_scale.fill_(old)
        check8(A, c, code, cache)
