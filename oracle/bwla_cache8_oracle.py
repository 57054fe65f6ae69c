"""Plain NumPy oracle (fp64) of a serving step around the attention: norms of heads, a cache of 8-bit codes with a scale for each page
and head, and the step's tables.  Test infrastructure only."""
from __future__ import annotations

import numpy as np

TOP = {"i8": 127.0, "e4m3": 448.0}


def norm(x, w=None, eps=1e-6, centered=False):
    """x (..., d)."""
    x = np.asarray(x, np.float64)
    if centered:
        x = x - x.mean(-1, keepdims=True)
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + np.float64(np.float32(eps)))
    return y if w is None else y * np.asarray(w, np.float64)


def step_of(code, y):
    """The distance of codes around numbers of this size."""
    if code == "i8":
        return np.ones_like(np.asarray(y, np.float64))
    a = np.maximum(np.abs(np.asarray(y, np.float64)), 2.0 ** -6)
    return 2.0 ** (np.floor(np.log2(a)) - 3)


def nearest(code, y):
    """Nearest code of each number, ties to even; what is too large becomes the largest, NaN 0."""
    y = np.clip(np.nan_to_num(np.asarray(y, np.float64), nan=0.0, posinf=1e300, neginf=-1e300), -TOP[code], TOP[code])
    step = step_of(code, y)
    return np.rint(y / step) * step


def grow(code, scale, most, fresh):
    """The scale behind new values of magnitude `most`, and how often the old one was doubled.  fresh: no older token lies in the page."""
    top = TOP[code]
    if fresh or not scale > 0:
        return (max(most / top, 2.0 ** -126) if most > 0 else 0.0), 0
    n, room = 0, float(np.float32(top) * np.float32(scale))    # (the product as fp32 has it: what once set a scale does not double it)
    while most > room * 2.0 ** n or (most > 0 and scale * 2.0 ** n < 2.0 ** -126):
        n += 1
    return scale * 2.0 ** n, n


def append(code, codes, scale, values, inside):
    """One page and head: codes (slots, d), its scale, values (tokens, d) of the new tokens behind `inside` older ones.  Changes codes;
    returns the scale and the number of doublings."""
    values = np.asarray(values, np.float64)
    finite = np.abs(values[np.isfinite(values)])
    was = scale
    scale, n = grow(code, scale, float(finite.max()) if finite.size else 0.0, inside == 0)
    if not was > 0 and scale > 0:
        codes[:inside] = 0                             # (what they stood for)
    if n:
        codes[:inside] = nearest(code, codes[:inside] / 2.0 ** n)
    with np.errstate(all="ignore"):
        codes[inside:inside + len(values)] = nearest(code, values / scale) if scale > 0 else 0.0
    return scale, n


def build(length, new, table, ring, state, page, pages, tokens, max_len, done=None, shift=None):
    """Returns a dict of what batch_build leaves.  table and ring are copied."""
    n_req = len(length)
    table, ring = np.array(table, np.int32), np.array(ring, np.int32)
    cap = len(ring)
    front, count = (int(state[0]) % 2 ** 32) % cap, int(np.clip(state[1], 0, cap))
    cut = np.clip(np.asarray(length, np.int64), 0, max_len)
    new = np.maximum(np.asarray(new, np.int64), 0)
    over = np.zeros(n_req, bool) if done is None else np.asarray(done) != 0
    kept = np.where(over, 0, cut)
    up = lambda n: -(-int(n) // page)  # noqa: E731
    take = [up(kept[b] + new[b]) - up(kept[b]) for b in range(n_req)]
    back = 0
    for b in range(n_req):
        if over[b]:
            for p in table[b, :up(cut[b])].copy():
                if 0 <= p < pages:
                    if back < cap - count:
                        ring[(front + count + back) % cap] = p
                    back += 1
    missing, long, rows = max(sum(take) - count, 0), int(sum(kept + new > max_len)), max(int(new.sum()) - tokens, 0)
    ok = missing == 0 and long == 0 and rows == 0
    position, slot, sequence = np.full(tokens, -1, np.int32), np.full(tokens, -1, np.int64), np.full(tokens, -1, np.int32)
    first, at, taken = [0], 0, 0
    for b in range(n_req):
        if ok:
            for e in range(up(kept[b]), up(kept[b] + new[b])):
                table[b, e] = ring[(front + taken) % cap]
                taken += 1
            for i in range(int(new[b])):
                j = int(kept[b]) + i
                p = int(table[b, j // page])
                position[at], sequence[at] = j + (0 if shift is None else int(shift[b])), b
                slot[at] = p * page + j % page if 0 <= p < pages else -1
                at += 1
        first.append(at)
    most = 2 ** 31 - 1
    return {"length": (kept + (new if ok else 0)).astype(np.int32), "table": table, "ring": ring, "first": np.array(first, np.int32),
            "state": np.array([(front + taken) % cap, count - taken + min(back, cap - count)], np.int32), "position": position, "slot": slot,
            "sequence": sequence, "status": np.array([min(missing, most), long, min(rows, most), min(int(new.sum()), most)], np.int32)}
