"""Plain NumPy oracle (fp64) of what lies between the q|k|v and the o projection: rotary positions, softmax attention
over a cache, sums of its weights, eviction by them.  Test infrastructure only; nothing here is paged, blocked or fused: a
sequence's keys and values are arrays of cached tokens, and the caller says which of them exist."""
from __future__ import annotations

import numpy as np


def rotate(x, cos, sin, position, sections, interleaved=False):
    """x (tokens, heads, d); cos, sin (positions, pairs); position (axes, tokens)."""
    x = np.array(x, np.float64)
    pairs = cos.shape[1]
    axis = np.repeat(np.arange(len(sections)), sections)
    assert len(axis) == pairs
    for t in range(x.shape[0]):
        for i in range(pairs):
            row = position[axis[i]][t]
            c, s = np.float64(cos[row, i]), np.float64(sin[row, i])
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, pairs + i)
            u, v = x[t, :, a].copy(), x[t, :, b].copy()
            x[t, :, a], x[t, :, b] = u * c - v * s, u * s + v * c
    return x


def seen(n, new, exists=None, window=0, prefix=0, doc=None, position=None):
    """(new, n) truth values: new token t (index n - new + t) sees cached token j; a negative index sees nothing."""
    i, j = np.arange(n - new, n)[:, None], np.arange(n)[None, :]
    p = np.arange(n) if position is None else np.asarray(position, np.int64)[:n]
    at = np.clip(i, 0, None)
    near = np.ones((new, n), bool) if window == 0 else p[at] - p[None, :] < window if n else np.ones((new, n), bool)
    ok = ((j <= i) & near) | (j < prefix)
    if doc is not None and n:
        d = np.asarray(doc)[:n]
        ok &= (d[at] == d[None, :]) & (d[at] >= 0)
    if exists is not None:
        ok &= np.asarray(exists, bool)[None, :n]
    return ok & (i >= 0)


def scores(q, k, scale, cap=0.0, slope=0.0, position=None):
    """One head: q (new, d), k (n, d)."""
    n, new = len(k), len(q)
    s = np.asarray(q, np.float64) @ np.asarray(k, np.float64).T * scale
    if cap:
        s = cap * np.tanh(s / cap)
    if slope and n:
        p = np.arange(n) if position is None else np.asarray(position, np.int64)[:n]
        i = np.clip(np.arange(n - new, n), 0, None)
        s = s - slope * np.abs(p[i][:, None] - p[None, :])
    return s


def softmax(s, ok):
    """Weights and logarithms of the sums over what is seen (0 and -inf where that is nothing)."""
    w, lse = np.zeros(s.shape), np.full(len(s), -np.inf)
    for t in range(len(s)):
        if ok[t].any():
            top = s[t][ok[t]].max()
            e = np.exp(s[t][ok[t]] - top)
            w[t][ok[t]] = e / e.sum()
            lse[t] = top + np.log(e.sum())
    return w, lse


def attend(q, k, v, scale, cap=0.0, slopes=None, window=0, prefix=0, doc=None, position=None, exists=None):
    """One sequence: q (new, hq, d), k and v (n, hkv, d).  Returns out (new, hq, d), lse (new, hq), the softmax weights
    summed over new tokens and a group's heads (n, hkv), and bounds of the error analysis: sum_j w |v| (like out) and,
    like lse, the largest scale sum_c |q_c k_c| and |score| of what a row sees."""
    new, hq, d = q.shape
    n, hkv = k.shape[:2]
    ok = seen(n, new, exists, window, prefix, doc, position)
    out, lse, sums = np.zeros((new, hq, d)), np.full((new, hq), -np.inf), np.zeros((n, hkv))
    vabs, qk, top = np.zeros((new, hq, d)), np.zeros((new, hq)), np.zeros((new, hq))
    some = ok.any(0)                                   # what no query sees may hold anything
    for h in range(hq):
        g = h // (hq // hkv)
        kg, vg = (np.where(some[:, None], np.asarray(x[:, g], np.float64), 0.0) for x in (k, v))
        s = scores(q[:, h], kg, scale, cap, 0.0 if slopes is None else float(slopes[h]), position)
        w, lse[:, h] = softmax(s, ok)
        out[:, h], vabs[:, h] = w @ vg, w @ np.abs(vg)
        sums[:, g] += w.sum(0)
        if n:
            qk[:, h] = np.where(ok, np.abs(np.asarray(q[:, h], np.float64)) @ np.abs(kg).T * scale, 0).max(1)
            top[:, h] = np.where(ok, np.abs(s), 0).max(1)
    return out, lse, sums, vabs, qk, top


def kept(weights, keep, sinks=0, recent=0, exists=None):
    """Indices of the tokens that stay.  weights (n, kv_heads) fp32."""
    n = len(weights)
    total = []
    for row in np.asarray(weights):
        x = np.float64(0)
        for w in row:
            x += np.float64(w)
        with np.errstate(over="ignore"):
            total.append(-np.inf if np.isnan(x) else float(np.float32(x)))
    there = [j for j in range(n) if exists is None or exists[j]]
    order = sorted(there, key=lambda j: (not (j < sinks or j >= n - recent), -total[j], j))
    return np.array(sorted(order[:keep]), np.int64)
