"""Values that attention calls get now and then: caps far above the scores, queries that are not numbers, calls that leave new
tokens out.  Oracle, cases and the bounds' derivation as in test_gpu_attention.py."""
import numpy as np
import pytest

from oracle import bwla_attention_oracle as orc
from test_gpu_attention import U, Case, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    pytest.importorskip("torch")                       # (in front of the library: one HIP runtime for both)
    from paper_2605_00422_amd import attention_binding
    attention_binding.load()
    return attention_binding


def run(c, A, score, batch=None):
    """out, lse, and the sums of weights of the same call (from 0) and of a call of their own (from 2)."""
    torch = c.torch
    cache, batch, q = A.KVCache(c.k, c.v), batch or c.batch(A), c.q.cuda()
    out, lse = torch.full_like(q, 9.0), torch.full((c.tokens, c.hq), 9.0, device="cuda")
    sums, alone = cache.weights(), cache.weights() + 2.0
    scratch = lambda n: torch.full((max(16, n),), 0xff, dtype=torch.uint8, device="cuda")  # noqa: E731
    A.attention_forward(cache, batch, score, q, out, lse, sums, scratch(A.attention_workspace_size(cache, batch, c.hq, True)))
    A.attention_weights(cache, batch, score, q, lse, alone, scratch(A.attention_weights_workspace_size(cache, batch, c.hq)))
    return out.float().cpu().numpy(), lse.cpu().numpy(), sums.cpu().numpy(), alone.cpu().numpy()


def of_tokens(c, sums, b):
    """(cached tokens, heads) of sequence b."""
    return np.array([sums[c.table_np[b, j // c.page], :, j % c.page] for j in range(c.lens[b])]).reshape(c.lens[b], c.hkv)


@pytest.mark.parametrize("cap", [127.0, 129.0, 1e3, 1e5, 1e7, 1e30])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,hq,hkv,lens,news", [(64, 6, 2, [190, 260], [190, 70]), (128, 8, 8, [300], [300]), (64, 8, 2, [900], [3]),
                                                (128, 4, 1, [1500], [40])])
def test_caps_far_above_the_scores(A, dtype, cap, d, hq, hkv, lens, news):
    """A cap is relative to the score: tanh(x) of a small x is x.  x = a scale / cap and C tanh(x) are six roundings, tanh itself is good to
    six units (below 0.6 to two): 16 U of the score.  bf16 up to a cap of 128: 8 U of the cap, which is 2^-14 at most."""
    c = Case(dtype, d, hq, hkv, 16, lens, news, seed=31)
    c.q = (c.q.float() * 4).to(c.T)                    # scores of +-30
    scale, bf = d ** -0.5, dtype == "bf16"
    out, lse, sums, alone = run(c, A, A.Score(scale, cap=cap))
    row = 0
    for b, (n, new) in enumerate(zip(lens, news)):
        k, v = (x.float().numpy() for x in c.kv[b])
        rows = slice(row, row + new)
        row += new
        want, want_lse, want_sums, vabs, qk, top = orc.attend(c.q[rows].float().numpy(), k, v, scale, cap=cap)
        eps = 2 * (d + 4) * U * qk + 16 * U * top + (8 * U * cap if bf and cap <= 128 else 0)
        rel = np.expm1(2 * eps) + (2 * n + 16) * U
        bound = vabs * (rel[..., None] + (2.0 ** -9 if bf else 0)) + np.abs(want) * (2.0 ** -8 if bf else 4 * U) + 1e-30
        assert np.all(np.abs(out[rows] - want) <= bound), np.max(np.abs(out[rows] - want) / bound)
        most = rel + 8 * U * (np.abs(want_lse) + 1)
        assert np.all(np.abs(lse[rows] - want_lse) <= most), np.max(np.abs(lse[rows] - want_lse) / most)
        most = want_sums * ((rel + 8 * U * (np.abs(want_lse) + top)).max() + (new * hq // hkv + 8) * U)
        assert np.all(np.abs(of_tokens(c, sums, b) - want_sums) <= most + 1e-35)
        assert np.all(np.abs(of_tokens(c, alone, b) - 2.0 - want_sums) <= most + 2 * U * (2.0 + want_sums))


NOT_NUMBERS = [float("nan"), float("inf")]


@pytest.mark.parametrize("value", NOT_NUMBERS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,hq,hkv,lens,news,pad", [(64, 4, 2, [200, 150], [200, 150], 10), (128, 8, 1, [300], [260], 3), (64, 8, 8, [400], [400], 70),
                                                    (64, 4, 2, [900], [100], 10), (256, 2, 2, [700], [300], 5), (64, 4, 2, [300, 40], [9, 4], 3)])
def test_padding_that_is_not_a_number(A, dtype, d, hq, hkv, lens, news, pad, value):
    """The last tokens belong to no document, and neither their queries nor their keys and values are numbers: zeros and -inf come out,
    and all other rows as if they were not there."""
    gone = {(b, j) for b, n in enumerate(lens) for j in range(n - pad, n)}
    c = Case(dtype, d, hq, hkv, 16, lens, news, seed=32, nan_tokens=gone)
    doc, ends = np.zeros((len(lens), max(lens)), np.int32), np.cumsum(news)
    for b, n in enumerate(lens):
        doc[b, n - pad:n] = -1
        c.q[ends[b] - pad:ends[b]] = value
    c.options = lambda rng, names: ({"doc": c.i32(doc)}, lambda b: {"doc": doc[b]})
    out = check(c, A)
    for end in ends:
        assert not out[end - pad:end].any()


@pytest.mark.parametrize("value", NOT_NUMBERS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,new,prefix", [(70, 75, 70), (130, 140, 128), (3, 5, 2)])
def test_rows_in_front_of_the_cache_that_are_not_numbers(A, dtype, n, new, prefix, value):
    """More new tokens than cached ones: the first see nothing, not the prefix either."""
    c = Case(dtype, 64, 4, 2, 16, [n], [new], seed=33)
    c.q[:new - n] = value
    c.options = lambda rng, names: ({"prefix": c.i32([prefix])}, lambda b: {"prefix": prefix})
    assert not check(c, A)[:new - n].any()


@pytest.mark.parametrize("value", NOT_NUMBERS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kw", [{}, {"window": 40}])
@pytest.mark.parametrize("d,hq,hkv,lens,news", [
    (64, 6, 2, [200, 33], [1, 1]), (64, 6, 2, [200, 33], [3, 2]),              # few rows, one part of the cache each
    (128, 8, 1, [6000], [2]), (64, 4, 4, [900, 700], [4, 3]),                  # ... and several parts
    (64, 4, 2, [230, 100], [230, 60]), (256, 2, 1, [130], [90]),               # many rows
    (128, 4, 1, [900, 300], [60, 40]), (64, 14, 2, [600], [600]),              # ... over parts of the cache
])
def test_queries_that_are_not_numbers(A, d, hq, hkv, lens, news, kw, dtype, value):
    """NaN comes out of the rows whose queries are not numbers, and in the sums of what these rows see; nothing else changes."""
    c = Case(dtype, d, hq, hkv, 16, lens, news, seed=34)
    bad, bf = [(news[0] // 2, hq - 1), (sum(news) - 1, 0)], dtype == "bf16"
    for row, head in bad:
        c.q[row, head] = value
    out, lse, sums, alone = run(c, A, A.Score(d ** -0.5, **kw))
    row = 0
    with np.errstate(invalid="ignore"):
        for b, (n, new) in enumerate(zip(lens, news)):
            k, v = (x.float().numpy() for x in c.kv[b])
            rows = slice(row, row + new)
            row += new
            want, want_lse, want_sums, vabs, qk, top = orc.attend(c.q[rows].float().numpy(), k, v, d ** -0.5, **kw)
            ok = ~np.isnan(want_lse)
            eps = 2 * (d + 4) * U * qk + 8 * U * top
            rel = np.expm1(2 * eps) + (2 * n + 16) * U
            bound = vabs * (rel[..., None] + (2.0 ** -9 if bf else 0)) + np.abs(want) * (2.0 ** -8 if bf else 4 * U) + 1e-30
            assert np.array_equal(np.isnan(lse[rows]), ~ok) and np.array_equal(np.isnan(out[rows]).all(-1), ~ok)
            assert np.all((np.abs(out[rows] - want) <= bound)[ok])
            assert np.all((np.abs(lse[rows] - want_lse) <= rel + 8 * U * (np.abs(want_lse) + 1))[ok])
            most = want_sums * ((rel + 8 * U * (np.abs(want_lse) + top))[ok].max(initial=0) + (new * hq // hkv + 8) * U)
            for got, extra in ((of_tokens(c, sums, b), 1e-35), (of_tokens(c, alone, b) - 2.0, 2 * U * (2.0 + want_sums))):
                assert np.array_equal(np.isnan(got), np.isnan(want_sums))
                assert np.all((np.abs(got - want_sums) <= most + extra)[~np.isnan(want_sums)])


# ---------------------------------------------------------------- more new tokens than the call takes
CUT = [  # (cached, new, max_new, rows of the call): sequences with more new tokens than max_new, or than there are rows
    ([200, 90, 33], [20, 3, 1], 4, 24), ([200, 90], [90, 60], 50, 150), ([600, 500], [300, 200], 130, 500), ([120, 100], [40, 30], 40, 60),
    ([9, 30], [20, 30], 15, 50), ([40, 40], [30, 10], 30, 30),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("prefix", [0, 150])
@pytest.mark.parametrize("lens,news,max_new,tokens", CUT)
def test_more_new_tokens_than_the_call_takes(A, dtype, prefix, lens, news, max_new, tokens):
    """The first of them come out as if all had been taken; the others' rows stay, and what is stored of them may be anything
    (in a prefix it is seen)."""
    first = np.concatenate([[0], np.cumsum(news)])
    taken = [max(0, min(new, max_new, tokens - int(r0))) for new, r0 in zip(news, first)]
    left = {(b, j) for b, n in enumerate(lens) for j in range(max(n - news[b] + taken[b], 0), n)} if not prefix else set()
    c = Case(dtype, 64, 4, 2, 16, lens, news, seed=35, nan_tokens=left)
    q, per = c.q, [min(prefix, n) for n in lens]
    c.q, c.tokens = q[:tokens], tokens
    score = A.Score(0.125, prefix=c.i32(per) if prefix else None)
    out, lse, sums, _ = run(c, A, score, c.batch(A, max_new=max_new))
    for b, (n, new) in enumerate(zip(lens, news)):
        rows = slice(int(first[b]), int(first[b]) + taken[b])
        rest = slice(rows.stop, min(int(first[b + 1]), tokens))
        assert (out[rest] == 9).all() and (lse[rest] == 9).all()
        if not taken[b]:
            continue
        k, v = (x.float().numpy() for x in c.kv[b])
        # all new rows (what the ones that are left out see does not matter), so that indexes are the sequence's
        doc = np.zeros(n, int)
        full = np.zeros((new, 4, 64), np.float32)
        full[:taken[b]] = c.q[rows].float().numpy()
        finite = lambda x: np.where(np.isfinite(x), x, 0)  # noqa: E731
        want, want_lse, _, vabs, qk, top = (x[:taken[b]] for x in orc.attend(full, finite(k), finite(v), 0.125, prefix=per[b], doc=doc))
        rel = np.expm1(4 * 68 * U * qk + 16 * U * top) + (2 * n + 16) * U
        bf = dtype == "bf16"
        bound = vabs * (rel[..., None] + (2.0 ** -9 if bf else 0)) + np.abs(want) * (2.0 ** -8 if bf else 4 * U) + 1e-30
        assert np.all(np.abs(out[rows] - want) <= bound), b
        some = ~np.isneginf(want_lse)
        assert np.array_equal(np.isneginf(lse[rows]), ~some)
        assert np.all((np.abs(lse[rows] - want_lse) <= rel + 8 * U * (np.abs(want_lse) + 1))[some])
        # each row that sees anything gives its tokens a weight of 1 in all, and heads of a group share a sum
        got = of_tokens(c, sums, b)
        assert np.all(np.abs(got.sum(0) - some.sum(0).reshape(2, 2).sum(1)) <= 1e-3 * taken[b])
        seen = max(n - new + taken[b], per[b], 0)
        assert not got[seen:].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rope_append_of_more_new_tokens_than_the_call_takes(A, dtype):
    import torch
    lens, news, max_new, tokens, hq, hkv, d, page = [40, 7, 25], [9, 1, 12], 4, 16, 4, 2, 64, 16
    c = Case(dtype, d, hq, hkv, page, lens, news, seed=36)
    first = np.concatenate([[0], np.cumsum(news)])
    c.tokens = tokens
    rope = A.Rope(torch.ones(50, 32, device="cuda"), torch.zeros(50, 32, device="cuda"))         # (turned by nothing)
    qkv = torch.randn(tokens, (hq + 2 * hkv) * d, device="cuda").to(c.T).float()
    pos = torch.arange(tokens, dtype=torch.int32, device="cuda")[None]
    q, cpos = torch.full((tokens, hq, d), 9.0, dtype=c.T, device="cuda"), torch.full((3, 40), -7, dtype=torch.int32, device="cuda")
    cache = A.KVCache(c.k, c.v)
    k, v, w = c.k.float().cpu().numpy(), c.v.float().cpu().numpy(), cache.weights() + 1.0
    A.rope_append(cache, c.batch(A, max_new=max_new), rope, qkv, pos, q, w, cpos)
    h, want_w, want_pos = qkv.cpu().numpy().reshape(tokens, -1, d), np.ones(tuple(w.shape)), np.full((3, 40), -7)
    want_q = np.full((tokens, hq, d), 9.0)
    for b, (n, new) in enumerate(zip(lens, news)):
        for t in range(min(new, max_new, tokens - int(first[b]))):
            row, j = int(first[b]) + t, n - new + t
            p, s = c.table_np[b, j // page], j % page
            want_q[row], k[p, :, s], v[p, :, s], want_w[p, :, s], want_pos[b, j] = h[row, :hq], h[row, hq:hq + hkv], h[row, hq + hkv:], 0, row
    assert np.array_equal(q.float().cpu().numpy(), want_q)
    assert np.array_equal(c.k.float().cpu().numpy(), k, equal_nan=True) and np.array_equal(c.v.float().cpu().numpy(), v, equal_nan=True)
    assert np.array_equal(w.cpu().numpy(), want_w) and np.array_equal(cpos.cpu().numpy(), want_pos)
