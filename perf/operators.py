"""The work that the attention half of a decoder block is measured on, next to the linear layers of cases.py.

The merged q|k|v projection of a quantized block leaves fp32 rows; the o projection reads bf16 (or fp32) rows.
Between them, over a key-value cache in pages:

  rope     attention_binding.rope_append: the rotary positions (one axis, or time/height/width) of the
           projection's rows, queries written dense, keys and values written to their pages
  attend   attention_binding.attention_forward: softmax attention of each sequence's new tokens (one, a chunk or a
           whole prompt) over its cache, with a cap by tanh, a bias by distance, a window, a prefix mask and a
           document mask; with "weights" it also adds each cached token's attention weight to its running sum
  weights  attention_binding.attention_weights: that sum on its own, for a prompt's queries
  evict    attention_binding.cache_evict: each sequence's heaviest tokens moved to pages of their own

Definition, for query t of sequence b (cache index i, position p) and cached token j (position r):

  seen(t, j)  = the page of j exists, doc[i] = doc[j] >= 0, and (j < prefix, or j <= i and p - r < window)
  s(t, j)     = capped(scale q_t . k_j) - slope_h |p - r|,   capped(x) = cap tanh(x / cap)
  w(t, j)     = exp(s(t, j) - lse_t) where seen, else 0,     lse_t = log sum_j exp s(t, j)
  out_t       = sum_j w(t, j) v_j  (0 where nothing is seen)

Head counts and sizes are those of the blocks in inputs.py and cases.py (4096 wide: 32 heads of 128, 32 or 8 key-value
heads; 5120: 40 and 8; 8192: 64 and 8; 2048: 16 and 4), and generic ones around them.
"""
import random

import numpy as np
import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _attend(name, op, x, hq, hkv, d, page, seqs, len_lo, len_hi, new, cap=0.0, slopes=False, window=0, prefix=0, docs=0,
            gone=0, weights=False, moved=False):
    """new: new tokens of the longest sequence (others have fewer where their cache holds fewer); docs: documents per sequence;
    gone: pages at the front of each sequence that were given back; moved: positions of cached tokens that are not their index."""
    return {"name": name, "op": op, "x": x, "hq": hq, "hkv": hkv, "d": d, "page": page, "seqs": seqs, "len_lo": len_lo,
            "len_hi": len_hi, "new": new, "cap": cap, "slopes": slopes, "window": window, "prefix": prefix, "docs": docs,
            "gone": gone, "weights": weights, "moved": moved}


def _rope(name, x, hq, hkv, d, page, seqs, new, rot, axes, pairs="halves", qkv="f32"):
    return {"name": name, "op": "rope", "x": x, "hq": hq, "hkv": hkv, "d": d, "page": page, "seqs": seqs, "len_lo": new,
            "len_hi": new + 4 * page, "new": new, "rot": rot, "axes": axes, "pairs": pairs, "qkv": qkv}


def _evict(name, x, hkv, d, page, seqs, len_lo, len_hi, keep, sinks, recent):
    return {"name": name, "op": "evict", "x": x, "hkv": hkv, "d": d, "page": page, "seqs": seqs, "len_lo": len_lo,
            "len_hi": len_hi, "keep": keep, "sinks": sinks, "recent": recent}


def listed():
    return [
        # one decoding step of sixteen sequences of a 5120-wide block: latency
        _rope("rope_step_m16", "bf16", 40, 8, 128, 16, 16, 1, 128, 1),
        # a prompt with images in it (time, height, width) through an 8192-wide block
        _rope("rope_axes_m4096", "bf16", 64, 8, 128, 64, 1, 4096, 128, 3),
        # the smallest attention: a few young sequences of a small fp32 model, latency
        _attend("decode_tiny_f32", "attend", "f32", 8, 8, 64, 16, 3, 1, 37, 1),
        # one sequence with a long cache, one new token: 8192-wide block
        _attend("decode_long_m1", "attend", "bf16", 64, 8, 128, 64, 1, 32768, 32768, 1),
        # a serving batch with caches of all ages, capped scores, weights summed for eviction
        _attend("decode_batch_m64", "attend", "bf16", 64, 8, 128, 16, 64, 500, 8192, 1, cap=50.0, weights=True),
        # a prompt of a 4096-wide block without shared heads, no options
        _attend("prompt_m2048", "attend", "bf16", 32, 32, 128, 16, 1, 2048, 2048, 2048),
        # documents packed into one long row, capped scores
        _attend("prompt_docs_m8192", "attend", "bf16", 32, 8, 128, 64, 1, 8192, 8192, 8192, cap=30.0, docs=5),
        # chunks of an odd size behind caches of several lengths, distance bias, a prefix seen by all
        _attend("chunk_m333", "attend", "bf16", 40, 8, 128, 16, 4, 900, 7001, 333, slopes=True, prefix=77),
        # weights of a small fp32 prompt
        _attend("weights_f32_m61", "weights", "f32", 16, 4, 128, 16, 2, 61, 117, 61),
        # weights that the last queries of long prompts give the prompt's tokens
        _attend("weights_m64", "weights", "bf16", 64, 8, 128, 64, 4, 6000, 16384, 64),
        # young sequences of a small model cut to a small budget: latency
        _evict("evict_small", "bf16", 4, 64, 16, 3, 300, 601, 256, 4, 32),
        # a batch of long sequences cut to a quarter
        _evict("evict_m16", "bf16", 8, 128, 64, 16, 9000, 16384, 4096, 4, 512),
    ]


_HEADS = [(32, 32), (64, 8), (40, 8), (32, 8), (16, 4), (8, 8), (16, 1), (6, 2), (12, 3)]
_MOST_BYTES = 1.1e9      # of cache that a drawn case reads
_MOST_PRODUCTS = 3.6e10  # pairs of a query and a key over all heads, times columns


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["rope", "attend", "attend", "attend", "attend", "weights", "evict"])
    x = "f32" if rng.random() < 0.25 else "bf16"
    size = 4 if x == "f32" else 2
    hq, hkv = rng.choice(_HEADS)
    d = rng.choice([128, 128, 128, 64, 64, 96, 80, 256])
    page = rng.choice([8, 16, 16, 32, 64, 128])
    if op == "rope":
        seqs = _log(rng, 1, 64)
        rot = d if rng.random() < 0.7 else d // 2
        c = _rope("", x, hq, hkv, d, page, seqs, max(1, _log(rng, 1, 8192) // seqs), rot, rng.choice([1, 1, 2, 3]),
                  rng.choice(["halves", "halves", "neighbours"]), rng.choice(["f32", "f32", "bf16"]))
        del c["name"]
        return c
    while True:
        seqs, hi = _log(rng, 1, 64), _log(rng, 4, 32768)
        lo = max(1, int(hi * rng.random()))
        if 2 * seqs * hi * hkv * d * size > (_MOST_BYTES / 2 if op == "evict" else _MOST_BYTES):
            continue
        if op == "evict":
            keep = max(1, int(hi * rng.uniform(0.1, 0.9)))
            c = _evict("", x, hkv, d, page, seqs, lo, hi, keep, min(keep // 4, 4), int(keep * rng.uniform(0.0, 0.5)))
            break
        new = 1 if op == "attend" and rng.random() < 0.45 else _log(rng, 1, min(hi, 8192))
        if seqs * hq * new * hi * d > (_MOST_PRODUCTS if x == "bf16" and op == "attend" else _MOST_PRODUCTS / 4):
            continue
        r = rng.random
        c = _attend("", op, x, hq, hkv, d, page, seqs, lo, hi, new,
                    cap=rng.choice([20.0, 30.0, 50.0]) if r() < 0.35 else 0.0, slopes=r() < 0.25,
                    window=_log(rng, 1, hi) if r() < 0.25 else 0, prefix=rng.randint(1, hi) if r() < 0.2 else 0,
                    docs=rng.randint(2, 9) if r() < 0.2 else 0, gone=1 if r() < 0.2 and lo > 4 * page else 0,
                    weights=op == "attend" and r() < 0.3, moved=r() < 0.15)
        break
    del c["name"]
    return c


# ---------------------------------------------------------------- what follows from a case alone
def _lengths(case):
    """Cached tokens of each sequence, from len_lo to len_hi in an order that is none; the last one is len_hi."""
    lo, hi, n = case["len_lo"], case["len_hi"], case["seqs"]
    return [hi - (hi - lo) * (b * 40503 % 65536) // 65536 for b in range(n)]


def _news(case):
    return [min(case["new"], n) for n in _lengths(case)]


def _docs(case, n):
    """Document of each of n cached tokens: runs of falling length, and the last token (padding) in none in prompts of five."""
    doc = np.floor(case["docs"] * ((np.arange(n) + 0.5) / n) ** 1.3).astype(np.int32)
    if case["docs"] == 5 and case["new"] > 1:
        doc[-1] = -1
    return doc


def _positions(case, n):
    """Positions of n cached tokens of which some were evicted: gaps of one in front."""
    i = np.arange(n, dtype=np.int32)
    return i + np.minimum(i, n // 2) if case["moved"] else i


def _seen_pairs(case):
    """Query-key pairs seen, over all sequences, and cached tokens that some query sees."""
    pairs = touched = 0
    for n, new in zip(_lengths(case), _news(case)):
        i, j = np.arange(n - new, n), np.arange(n)
        p, doc = _positions(case, n), _docs(case, n) if case["docs"] else np.zeros(n, np.int32)
        any_seen = np.zeros(n, bool)
        for at in range(0, new, 512):
            q = i[at:at + 512, None]
            seen = j <= q
            if case["window"]:
                seen &= p[q] - p[None, :] < case["window"]
            seen |= j < case["prefix"]
            seen &= (doc[q] == doc[None, :]) & (doc[q] >= 0) & (j >= case["gone"] * case["page"])
            pairs += int(seen.sum())
            any_seen |= seen.any(0)
        touched += int(any_seen.sum())
    return pairs, touched


def work(case):
    size = 4 if case["x"] == "f32" else 2
    if case["op"] == "rope":
        rows, width = sum(_news(case)), (case["hq"] + 2 * case["hkv"]) * case["d"]
        table = min(rows * case["axes"], case["len_hi"]) * case["rot"] * 4
        return {"bytes": rows * (width * (size + (4 if case["qkv"] == "f32" else 2)) + 4 * case["axes"]) + table,
                "flops": rows * (case["hq"] + case["hkv"]) * case["rot"] * 3}
    row = case["hkv"] * case["d"] * size
    if case["op"] == "evict":
        kept = sum(min(case["keep"], n) for n in _lengths(case))
        return {"bytes": sum(_lengths(case)) * case["hkv"] * 4 + kept * (4 * row + 4 * case["hkv"] + 12), "flops": 0}
    pairs, touched = _seen_pairs(case)
    q = sum(_news(case)) * case["hq"]
    sums = 2 * 4 * touched * case["hkv"]
    if case["op"] == "weights":
        return {"bytes": touched * row + q * (case["d"] * size + 4) + sums, "flops": 2 * pairs * case["hq"] * case["d"]}
    return {"bytes": 2 * touched * row + q * (2 * case["d"] * size + 4) + (sums if case["weights"] else 0),
            "flops": 4 * pairs * case["hq"] * case["d"]}


# ---------------------------------------------------------------- inputs
def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op, x, d, page, hkv, seqs = case["op"], _TYPES[case["x"]], case["d"], case["page"], case["hkv"], case["seqs"]
    lens = _lengths(case)
    per = -(-max(lens) // page)
    per_out = -(-case["keep"] // page) if op == "evict" else 0
    pages = seqs * (per + per_out) + 3
    draws = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    k, v = (torch.empty(pages, hkv, page, d, dtype=x, device="cuda") for _ in range(2))
    for t in (k, v):                     # keys with a few strong channels, as trained ones have
        for at in range(0, pages, 4096):
            t[at:at + 4096] = draws(*t[at:at + 4096].shape)
    k[..., :: max(1, d // 4)] *= 3.0
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = order[:seqs * per].reshape(seqs, per).contiguous()
    st = {"case": dict(case), "op": op, "k": k, "v": v, "table": table, "length": ints(lens), "lens": lens, "max_len": max(lens)}
    if op == "evict":
        # sums of weights: a few heavy tokens, many light ones, and equal ones among them
        st["weights"] = torch.floor(torch.exp(2 * draws(pages, hkv, page)) * 64) / 64
        st["table_out"] = order[seqs * per:seqs * (per + per_out)].reshape(seqs, per_out).contiguous()
        st["position"] = torch.arange(max(lens), device="cuda", dtype=torch.int32).repeat(seqs, 1) * 2 + 1
        st["position_out"] = torch.full((seqs, case["keep"]), -1, dtype=torch.int32, device="cuda")
        st["kept"] = torch.full((seqs, case["keep"]), -1, dtype=torch.int32, device="cuda")
        st["length_out"] = torch.zeros(seqs, dtype=torch.int32, device="cuda")
    else:
        news = _news(case)
        first = np.concatenate([[0], np.cumsum(news)])
        st |= {"tokens": int(first[-1]), "max_new": max(news), "first": ints(first.tolist()) if max(news) > 1 else None}
    if op == "rope":
        st["qkv"] = draws(st["tokens"], (case["hq"] + 2 * hkv) * d).to(_TYPES[case["qkv"]])
        n, pairs = max(lens) + 1, case["rot"] // 2
        angle = torch.arange(n, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (
            -torch.arange(pairs, device="cuda", dtype=torch.float64) / pairs)
        st["cos"], st["sin"] = angle.cos().float(), angle.sin().float()
        st["position"] = torch.randint(0, n, (case["axes"], st["tokens"]), generator=g, device="cuda", dtype=torch.int32)
        a, rest = case["axes"], pairs
        st["sections"] = [rest] if a == 1 else [pairs // 4] + [(pairs - pairs // 4) // (a - 1)] * (a - 2)
        st["sections"] += [pairs - sum(st["sections"])] if a > 1 else []
        st["q"] = torch.zeros(st["tokens"], case["hq"], d, dtype=x, device="cuda")
    elif op != "evict":
        st["q"] = (1.5 * draws(st["tokens"], case["hq"], d)).to(x)
        st["scale"] = d ** -0.5
        st["slopes"] = 2.0 ** (-8.0 * torch.arange(1, case["hq"] + 1, device="cuda") / case["hq"]) if case["slopes"] else None
        st["prefix"] = ints([min(case["prefix"], n) for n in lens]) if case["prefix"] else None
        row = lambda f: torch.from_numpy(np.stack([np.pad(f(case, n), (0, max(lens) - n)) for n in lens])).cuda()  # noqa: E731
        st["doc"] = row(_docs) if case["docs"] else None
        st["position"] = row(_positions) if case["moved"] else None
        if case["gone"]:
            table[:, :case["gone"]] = -1
        st["lse"] = torch.zeros(st["tokens"], case["hq"], device="cuda")
        st["out"] = torch.zeros_like(st["q"])
        st["weights"] = torch.zeros(pages, hkv, page, device="cuda") if case["weights"] or op == "weights" else None
        if op == "weights":                # the forward pass of these queries left it
            s = _scores(st)
            st["lse"].copy_(_softmax(s)[1][_rows(st)])
    if own:                                # what a serving program makes once: descriptors and a workspace
        from paper_2605_00422_amd import attention_binding as A
        st["cache"] = A.KVCache(k, v)
        if op == "evict":
            st["batch"] = A.Batch(table, st["length"], max_len=st["max_len"])
            n = A.cache_evict_workspace_size(st["cache"], st["batch"])
        else:
            st["batch"] = A.Batch(table, st["length"], st["first"], tokens=st["tokens"], max_new=st["max_new"], max_len=st["max_len"])
            n = 0
        if op == "rope":
            st["rope"] = A.Rope(st["cos"], st["sin"], st["sections"], interleaved=case["pairs"] == "neighbours")
        elif op != "evict":
            st["score"] = A.Score(st["scale"], cap=case["cap"], slopes=st["slopes"], window=case["window"], prefix=st["prefix"],
                                  doc=st["doc"], position=st["position"])
            if op == "attend":
                n = A.attention_workspace_size(st["cache"], st["batch"], case["hq"], case["weights"])
            else:
                n = A.attention_weights_workspace_size(st["cache"], st["batch"], case["hq"])
        st["ws"] = torch.zeros(max(n, 16), dtype=torch.uint8, device="cuda")
    return st


# ---------------------------------------------------------------- one pass
def run(st):
    if own:
        return _run_own(st)
    return {"rope": _plain_rope, "attend": _plain_attend, "weights": _plain_weights, "evict": _plain_evict}[st["op"]](st)


def _run_own(st):
    from paper_2605_00422_amd import attention_binding as A
    op = st["op"]
    if op == "rope":
        A.rope_append(st["cache"], st["batch"], st["rope"], st["qkv"], st["position"], st["q"])
        return {"q": st["q"], "k": st["k"], "v": st["v"]}
    if op == "attend":
        A.attention_forward(st["cache"], st["batch"], st["score"], st["q"], st["out"], st["lse"], st["weights"], st["ws"])
        return {"out": st["out"], "lse": st["lse"], "weights": st["weights"]}
    if op == "weights":
        A.attention_weights(st["cache"], st["batch"], st["score"], st["q"], st["lse"], st["weights"], st["ws"])
        return {"weights": st["weights"]}
    A.cache_evict(st["cache"], st["batch"], st["table_out"], st["weights"], st["case"]["keep"], st["case"]["sinks"],
                  st["case"]["recent"], st["length_out"], st["kept"], st["position"], st["position_out"], st["ws"])
    return {"k": st["k"], "v": st["v"], "weights": st["weights"], "kept": st["kept"], "length": st["length_out"],
            "position": st["position_out"]}


# the plain forms: torch's elementary operations, in 32 bits, rounded once at the end
def _rows(st):
    """(sequence, number among its new tokens) of each row of q."""
    b, n = st["table"].shape[0], st["tokens"]
    t = torch.arange(n, device="cuda")
    if st["first"] is None:
        return t, torch.zeros_like(t)
    s = torch.searchsorted(st["first"][1:b + 1].long().contiguous(), t, right=True)
    return s, t - st["first"].long()[s]


def _new(st):
    return torch.ones_like(st["length"]) if st["first"] is None else st["first"][1:] - st["first"][:-1]


def _gather(pool, st):
    """Sequences x heads x tokens x columns in fp32, of the pages that the table lists."""
    x = pool[st["table"].clamp(min=0).long()]
    b, p, h, s, d = x.shape
    return x.permute(0, 2, 1, 3, 4).reshape(b, h, p * s, d)[:, :, :st["max_len"]].float()


def _seen(st):
    c, page = st["case"], st["k"].shape[2]
    j = torch.arange(st["max_len"], device="cuda")
    i = (st["length"] - _new(st)).long()[:, None] + torch.arange(st["max_new"], device="cuda")
    there = (j < st["length"][:, None]) & (st["table"] >= 0).repeat_interleave(page, 1)[:, :st["max_len"]]
    i = i.clamp(max=st["max_len"] - 1)
    pos = j.expand(len(i), -1) if st["position"] is None else st["position"].long()
    apart = pos.gather(1, i)[:, :, None] - pos[:, None, :]
    seen = j <= i[:, :, None]
    if c["window"]:
        seen = seen & (apart < c["window"])
    if st["prefix"] is not None:
        seen = seen | (j < st["prefix"][:, None])[:, None, :]
    if st["doc"] is not None:
        mine = st["doc"].gather(1, i)[:, :, None]
        seen = seen & (mine == st["doc"][:, None, :]) & (mine >= 0)
    return seen & there[:, None, :], apart


def _scores(st):
    """Sequences x new tokens x heads x cached tokens, -inf where nothing is seen."""
    c = st["case"]
    b, m, hq, hkv, d = len(st["length"]), st["max_new"], c["hq"], c["hkv"], c["d"]
    q = torch.zeros(b, m, hq, d, device="cuda")
    q[_rows(st)] = st["q"].float()
    q = q.reshape(b, m, hkv, hq // hkv, d).permute(0, 2, 1, 3, 4).reshape(b, hkv, m * hq // hkv, d)
    s = torch.matmul(q, _gather(st["k"], st).transpose(-1, -2).contiguous()) * st["scale"]
    s = s.reshape(b, hkv, m, hq // hkv, -1).transpose(1, 2).reshape(b, m, hq, -1)
    if c["cap"]:
        s = c["cap"] * torch.tanh(s / c["cap"])
    seen, apart = _seen(st)
    if st["slopes"] is not None:
        s = s - st["slopes"][:, None] * apart.abs().float()[:, :, None, :]
    return s.masked_fill(~seen[:, :, None, :], float("-inf"))


def _softmax(s):
    """Weights and logarithms of their sums; rows that see nothing: 0 and -inf."""
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    lse = torch.where(torch.isinf(top), top, top + torch.log(total))
    return p / torch.where(total > 0, total, torch.ones_like(total)), lse[..., 0]


def _add_weights(st, p):
    """Sums over a sequence's new tokens and the heads of a group, added where the cached tokens lie."""
    b, m, hq, n = p.shape
    hkv, page = st["k"].shape[1:3]
    w = p.sum(1).reshape(b, hkv, hq // hkv, n).sum(2)
    j = torch.arange(n, device="cuda")
    at = st["table"].long()[:, j // page]
    ok = (at >= 0) & (j < st["length"][:, None])
    bi, ji = torch.where(ok)
    st["weights"][at[bi, ji], :, ji % page] += w[bi, :, ji]


def _plain_attend(st):
    p, lse = _softmax(_scores(st))
    b, m, hq, n = p.shape
    hkv = st["k"].shape[1]
    g = p.reshape(b, m, hkv, hq // hkv, n).transpose(1, 2).reshape(b, hkv, m * hq // hkv, n)
    at = torch.arange(n, device="cuda") < st["length"][:, None]
    v = _gather(st["v"], st).masked_fill(~at[:, None, :, None], 0.0)
    out = torch.matmul(g, v).reshape(b, hkv, m, hq // hkv, -1).transpose(1, 2).reshape(b, m, hq, -1)
    rows = _rows(st)
    st["out"].copy_(out[rows])
    st["lse"].copy_(lse[rows])
    if st["weights"] is not None:
        live = torch.arange(m, device="cuda") < _new(st)[:, None]
        _add_weights(st, p * live[:, :, None, None])
    return {"out": st["out"], "lse": st["lse"], "weights": st["weights"]}


def _plain_weights(st):
    lse = torch.full((len(st["length"]), st["max_new"], st["case"]["hq"]), float("inf"), device="cuda")
    lse[_rows(st)] = torch.where(torch.isinf(st["lse"]), -st["lse"], st["lse"])     # a row that sees nothing adds nothing
    _add_weights(st, torch.exp(_scores(st) - lse[..., None]))
    return {"weights": st["weights"]}


def _plain_rope(st):
    c = st["case"]
    hq, hkv, d, rot, n = c["hq"], c["hkv"], c["d"], c["rot"], st["tokens"]
    x = st["qkv"].float().reshape(n, hq + 2 * hkv, d)
    axis = torch.repeat_interleave(torch.arange(c["axes"], device="cuda"), torch.tensor(st["sections"], device="cuda"))
    pair = torch.arange(rot // 2, device="cuda")
    at = st["position"].long()[axis].T
    cos, sin = st["cos"][at, pair][:, None], st["sin"][at, pair][:, None]
    turned, qk = x.clone(), x[:, :hq + hkv, :rot]
    if c["pairs"] == "neighbours":
        a, b = qk[..., 0::2], qk[..., 1::2]
        turned[:, :hq + hkv, :rot] = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = qk[..., :rot // 2], qk[..., rot // 2:]
        turned[:, :hq + hkv, :rot] = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    s, i = _rows(st)
    j = (st["length"] - _new(st)).long()[s] + i
    at, slot = st["table"].long()[s, j // c["page"]], j % c["page"]
    st["q"].copy_(turned[:, :hq])
    st["k"][at, :, slot] = turned[:, hq:hq + hkv].to(st["k"].dtype)
    st["v"][at, :, slot] = turned[:, hq + hkv:].to(st["v"].dtype)
    return {"q": st["q"], "k": st["k"], "v": st["v"]}


def _plain_evict(st):
    c, page = st["case"], st["k"].shape[2]
    j, keep = torch.arange(st["max_len"], device="cuda"), c["keep"]
    at, slot = st["table"].long()[:, j // page], j % page
    n = st["length"].long()[:, None]
    w = st["weights"][at, :, slot].double().sum(-1).float()
    w = torch.where((j < c["sinks"]) | (j >= n - c["recent"]), torch.full_like(w, float("inf")), w)
    w = torch.where(j < n, w, torch.full_like(w, float("-inf")))
    first = torch.sort(w, dim=1, descending=True, stable=True)[1][:, :keep]
    count = torch.minimum(n, torch.full_like(n, keep))
    live = torch.arange(first.shape[1], device="cuda") < count
    kept = torch.sort(torch.where(live, first, torch.full_like(first, 1 << 30)), dim=1)[0]
    b, r = torch.where(live)
    frm, to = kept[b, r], st["table_out"].long()[b, r // page]
    st["kept"].fill_(-1)
    st["kept"][b, r] = frm.int()
    st["position_out"].fill_(-1)
    st["position_out"][b, r] = st["position"][b, frm]
    st["length_out"].copy_(count[:, 0])
    for pool in (st["k"], st["v"], st["weights"]):
        pool[to, :, r % page] = pool[at[b, frm], :, frm % page]
    return {"k": st["k"], "v": st["v"], "weights": st["weights"], "kept": st["kept"], "length": st["length_out"],
            "position": st["position_out"]}


# ---------------------------------------------------------------- the definition in 64 bits, one sequence and head at a time
def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "evict":
        return _exact_evict(st)
    if case["op"] == "rope":
        return _exact_rope(st)
    hq, hkv, page, op = case["hq"], case["hkv"], case["page"], case["op"]
    out, lse = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda"), torch.zeros(st["lse"].shape, dtype=torch.float64, device="cuda")
    sums = torch.zeros(st["k"].shape[:3], dtype=torch.float64, device="cuda")
    row = 0
    for b, (n, new) in enumerate(zip(_lengths(case), _news(case))):
        j = torch.arange(n, device="cuda")
        pages = st["table"][b].long()[j // page]
        p = torch.from_numpy(_positions(case, n)).cuda().long()
        doc = torch.from_numpy(_docs(case, n)).cuda() if case["docs"] else torch.zeros(n, device="cuda")
        prefix = 0 if st["prefix"] is None else int(st["prefix"][b])
        for h in range(hkv):
            k, v = (st[name][pages.clamp(min=0), h, j % page].double() for name in ("k", "v"))
            for at in range(0, new, 2048):
                i = torch.arange(n - new + at, min(n - new + at + 2048, n), device="cuda")
                rows = slice(row + at, row + at + len(i))
                apart = p[i][:, None] - p[None, :]
                allowed = j[None, :] <= i[:, None]
                if case["window"] > 0:
                    allowed = torch.logical_and(allowed, apart < case["window"])
                allowed = torch.logical_or(allowed, (j < prefix)[None, :])
                allowed = allowed & (doc[i][:, None] == doc[None, :]) & (doc[i][:, None] >= 0) & (pages >= 0)[None, :]
                for head in range(h * (hq // hkv), (h + 1) * (hq // hkv)):
                    s = st["q"][rows, head].double() @ k.T * st["scale"]
                    if case["cap"] > 0:
                        s = torch.tanh(s / case["cap"]) * case["cap"]
                    if st["slopes"] is not None:
                        s = s - st["slopes"][head].double() * apart.abs()
                    e = torch.where(allowed, torch.exp(s), torch.zeros((), dtype=torch.float64, device="cuda"))
                    total = e.sum(1)
                    if op == "weights":    # with the fp32 logarithms that the call is given
                        w = e * torch.exp(-st["lse"][rows, head].double().clamp(min=-700))[:, None]
                    else:
                        w = e / total.clamp(min=1e-300)[:, None]
                        out[rows, head] = w @ v
                        lse[rows, head] = torch.log(total)
                    sums[pages.clamp(min=0), h, j % page] += torch.where(pages >= 0, w.sum(0), torch.zeros_like(w[0]))
        row += new
    if op == "weights":
        return {"weights": sums}
    return {"out": out, "lse": lse, "weights": sums if case["weights"] else None}


def _exact_rope(st):
    c = st["case"]
    q, (k, v) = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda"), (st[n].double() for n in ("k", "v"))
    x = st["qkv"].double().reshape(st["tokens"], -1, c["d"])
    half, axis = c["rot"] // 2, sum(([a] * n for a, n in enumerate(st["sections"])), [])
    for i in range(half):
        lo, hi = (2 * i, 2 * i + 1) if c["pairs"] == "neighbours" else (i, half + i)
        at = st["position"][axis[i]].long()
        z = torch.complex(st["cos"][at, i].double(), st["sin"][at, i].double())[:, None]
        w = torch.complex(x[:, :c["hq"] + c["hkv"], lo], x[:, :c["hq"] + c["hkv"], hi]) * z
        x[:, :c["hq"] + c["hkv"], lo], x[:, :c["hq"] + c["hkv"], hi] = w.real, w.imag
    q.copy_(x[:, :c["hq"]])
    row = 0
    for b, (n, new) in enumerate(zip(_lengths(c), _news(c))):
        j = torch.arange(n - new, n, device="cuda")
        page = st["table"][b].long()[j // c["page"]]
        k[page, :, j % c["page"]] = x[row:row + new, c["hq"]:c["hq"] + c["hkv"]]
        v[page, :, j % c["page"]] = x[row:row + new, c["hq"] + c["hkv"]:]
        row += new
    return {"q": q, "k": k, "v": v}


def _exact_evict(st):
    c, page = st["case"], st["case"]["page"]
    k, v, w = (st[n].double() for n in ("k", "v", "weights"))
    kept, pos = np.full((c["seqs"], c["keep"]), -1, np.int32), np.full((c["seqs"], c["keep"]), -1, np.int32)
    for b, n in enumerate(_lengths(c)):
        j = torch.arange(n, device="cuda")
        pages = st["table"][b].long()[j // page]
        total = w[pages, :, j % page].sum(1).float().cpu().numpy()
        order = sorted(range(n), key=lambda i: (not (i < c["sinks"] or i >= n - c["recent"]), -float(total[i]), i))
        mine = np.array(sorted(order[:c["keep"]]))
        kept[b, :len(mine)], pos[b, :len(mine)] = mine, 2 * mine + 1
        mine = torch.from_numpy(mine).cuda()
        r = torch.arange(len(mine), device="cuda")
        to = st["table_out"][b].long()[r // page]
        for pool in (k, v, w):
            pool[to, :, r % page] = pool[pages[mine], :, mine % page]
    return {"k": k, "v": v, "weights": w, "kept": kept, "length": np.minimum(_lengths(c), c["keep"]).astype(np.int32), "position": pos}


if __name__ == "__main__":
    for c in listed() + [draw(random.Random(s)) for s in range(4)]:
        print(c.get("name", "drawn"), work(c))
