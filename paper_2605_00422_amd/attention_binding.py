"""ctypes binding of what lies between the q|k|v and the o projection (include/bwla.h): norms of the heads, rotary positions, the
paged key-value cache (as it is or in 8 bits), attention over it, eviction from it, and a step's tables.  The same names without the `bwla_` prefix, argument marshalling
only; every step runs in the library's HIP kernels.  Device arrays are torch CUDA tensors; the descriptors KVCache, KVCache8,
Batch, Score, Rope, HeadNorm and PagePool hold their tensors, whose contents may change between calls (a serving loop makes them once)."""
from __future__ import annotations

from ctypes import POINTER, Structure, byref, c_float, c_int, c_int32, c_int64, c_size_t, c_void_p

from . import binding as _b


class _Cache(Structure):
    _fields_ = [("d_k", c_void_p), ("d_v", c_void_p), ("page_stride", c_int64), ("head_stride", c_int64), ("slot_stride", c_int64),
                ("pages", c_int64), ("page_size", c_int32), ("kv_heads", c_int32), ("head_dim", c_int32), ("dtype", c_int32)]


class _Batch(Structure):
    _fields_ = [("d_table", c_void_p), ("d_len", c_void_p), ("d_first", c_void_p), ("tokens", c_int64), ("sequences", c_int32),
                ("table_stride", c_int32), ("max_new", c_int32), ("max_len", c_int32)]


class _Score(Structure):
    _fields_ = [("d_slopes", c_void_p), ("d_prefix", c_void_p), ("d_doc", c_void_p), ("d_position", c_void_p), ("scale", c_float),
                ("cap", c_float), ("window", c_int32), ("index_stride", c_int32)]


class _Rope(Structure):
    _fields_ = [("d_cos", c_void_p), ("d_sin", c_void_p), ("rows", c_int32), ("pairs", c_int32),
                ("axes", c_int32), ("interleaved", c_int32), ("sections", c_int32 * 4)]


class _Cache8(Structure):
    _fields_ = [("d_k", c_void_p), ("d_v", c_void_p), ("d_k_scale", c_void_p), ("d_v_scale", c_void_p), ("page_stride", c_int64),
                ("head_stride", c_int64), ("slot_stride", c_int64), ("scale_stride", c_int64), ("pages", c_int64), ("page_size", c_int32),
                ("kv_heads", c_int32), ("head_dim", c_int32), ("code", c_int32), ("dtype", c_int32)]


class _HeadNorm(Structure):
    _fields_ = [("d_q", c_void_p), ("d_k", c_void_p), ("q_stride", c_int64), ("k_stride", c_int64), ("eps", c_float), ("centered", c_int32)]


class _Pool(Structure):
    _fields_ = [("d_ring", c_void_p), ("d_state", c_void_p), ("d_state_out", c_void_p), ("pages", c_int64), ("capacity", c_int32),
                ("page_size", c_int32)]


CODE_I8, CODE_E4M3 = 0, 1
_lib = None


def load():
    global _lib
    if _lib is not None:
        return _lib
    lib = _b.load()
    P, I32, I64, SZ = c_void_p, c_int32, c_int64, c_size_t
    lib.bwla_rope_append.argtypes = [P, P, P, P, P, c_int, I64, I32, P, P, P, I32, P]
    lib.bwla_attention_workspace_size.argtypes = [P, P, I32, c_int, POINTER(c_size_t)]
    lib.bwla_attention_forward.argtypes = [P, P, P, P, I64, I32, P, P, P, P, SZ, P]
    lib.bwla_attention_weights_workspace_size.argtypes = [P, P, I32, POINTER(c_size_t)]
    lib.bwla_attention_weights.argtypes = [P, P, P, P, I64, I32, P, P, P, SZ, P]
    lib.bwla_cache_evict_workspace_size.argtypes = [P, P, POINTER(c_size_t)]
    lib.bwla_cache_evict.argtypes = [P, P, P, I32, P, I32, I32, I32, P, P, P, I32, P, P, SZ, P]
    lib.bwla_norm_rope_append.argtypes = [P, P, P, P, P, P, c_int, I64, I32, P, P, P, I32, P]
    lib.bwla_norm_rope_append8.argtypes = [P, P, P, P, P, P, c_int, I64, I32, P, P, I32, P]
    lib.bwla_cache8_read.argtypes = [P, P, P, P, c_int, P]
    lib.bwla_attention8_workspace_size.argtypes = [P, P, I32, POINTER(c_size_t)]
    lib.bwla_attention8_forward.argtypes = [P, P, P, P, I64, I32, P, P, P, SZ, P]
    lib.bwla_batch_build_workspace_size.argtypes = [I32, I64, POINTER(c_size_t)]
    lib.bwla_batch_build.argtypes = [P, P, P, P, P, P, I32, I32, I64, I32, P, P, P, P, P, P, P, SZ, P]
    _lib = lib
    return lib


_p, _s, _ck = _b._ptr, _b._stream, _b._check
_i32 = _f32 = _i64 = None


# The checks of a call take as long on the host as a small call on the GPU: shapes and strides are read once each, and what a
# descriptor knows is looked up there (16 rows of 40 heads: rope_append 7.0 -> 3.7 us, attention_forward 7.8 -> 4.2 us).
def _types():
    global _i32, _f32, _i64
    if _i32 is None:
        import torch
        _i32, _f32, _i64 = torch.int32, torch.float32, torch.int64


def _bytes(t) -> int:
    return 0 if t is None else t.nbytes


def _ints(t, what: str, dims: int):
    """A dense int32 tensor of so many dimensions (rows may be apart), or None."""
    if t is not None and (t.dtype is not _i32 or t.dim() != dims or (t.stride()[-1] != 1 and t.shape[-1] > 1 and t.numel())):
        raise TypeError(f"{what} must be an int32 tensor of {dims} dimensions, contiguous in the last")
    return t


def _floats(t, what: str, shape=None):
    if t is not None and (t.dtype is not _f32 or (shape is not None and t.shape != shape) or not t.is_contiguous()):
        raise TypeError(f"{what} must be a contiguous float32 tensor" + (f" of shape {tuple(shape)}" if shape is not None else ""))
    return t


def _on(*tensors):
    """Index of the GPU that these tensors lie on (-1: none of them on one), None without any, -2 where they lie apart."""
    at = {t.get_device() for t in tensors if t is not None}
    return None if not at else at.pop() if len(at) == 1 else -2


class KVCache:
    """Keys and values in pages: two tensors (pages, kv_heads, page_size, head_dim), float32 or bfloat16, of any strides
    (the same for both) with dense columns."""

    def __init__(self, k, v):
        if k.dim() != 4 or k.shape != v.shape or k.stride() != v.stride() or k.dtype != v.dtype:
            raise TypeError("k and v must be alike: (pages, kv_heads, page_size, head_dim)")
        if k.stride(3) != 1 and k.shape[3] > 1:
            raise TypeError("a head's columns must be dense")
        _types()
        self.k, self.v, self.dtype, self._at = k, v, k.dtype, _on(k, v)
        self.slots = k.shape[:3]
        self.pages, self.kv_heads, self.page_size, self.head_dim = k.shape
        self.desc = _Cache(_p(k), _p(v), k.stride(0), k.stride(1), k.stride(2), *k.shape[:1], k.shape[2], k.shape[1], k.shape[3],
                           _b._xdtype(k))
        self._ref = byref(self.desc)

    def weights(self):
        """Sums of attention weights for this cache, zero."""
        import torch
        return torch.zeros(self.pages, self.kv_heads, self.page_size, dtype=torch.float32, device=self.k.device)

    def _of(self, t, what):
        return _floats(t, what, self.slots)


class Batch:
    """The sequences of a call.  table (sequences, pages of the longest) and length (sequences): int32.  first (sequences + 1): the
    new tokens' rows, or None: one new token each.  tokens, max_new (both with `first`), max_len: rows of the call, most new and most
    cached tokens of a sequence, known on the host (the tensors are not read here)."""

    def __init__(self, table, length, first=None, tokens=None, max_new=None, max_len=None):
        _types()
        self.table, self.length, self.first = _ints(table, "table", 2), _ints(length, "length", 1), _ints(first, "first", 1)
        n = length.shape[0]
        if table.shape[0] != n or (first is not None and first.shape[0] != n + 1):
            raise ValueError("table, length and first belong to different numbers of sequences")
        if first is not None and tokens is None:
            raise ValueError("tokens: the rows of the call")
        if first is not None and max_new is None:
            raise ValueError("max_new: the most new tokens of a sequence")
        if max_len is None:
            raise ValueError("max_len: the most cached tokens of a sequence")
        self._at = _on(table, length, first)
        self.sequences, self.tokens = n, int(n if tokens is None else tokens)
        self.max_len, self.columns = int(max_len), table.shape[1]
        stride = table.stride(0) if n > 1 else table.shape[1]
        if stride < table.shape[1]:
            raise TypeError("rows of the table overlap")
        self.desc = _Batch(_p(table), _p(length), _p(first), self.tokens, n, stride, 1 if max_new is None else int(max_new), self.max_len)
        self._ref = byref(self.desc)

    # (The library knows the distance of rows, not how much of it belongs to them: a view may be narrower.)
    def _fits(self, cache):
        if self.columns * cache.page_size < self.max_len:
            raise ValueError("table: too few pages for max_len")


class Score:
    """How a query and a key make a score, and what a query sees: bwla_score_t."""

    def __init__(self, scale, cap=0.0, slopes=None, window=0, prefix=None, doc=None, position=None):
        _types()
        self.slopes, self.prefix = _floats(slopes, "slopes"), _ints(prefix, "prefix", 1)
        self.doc, self.position = _ints(doc, "doc", 2), _ints(position, "position", 2)
        self.heads, self._at = None if slopes is None else slopes.numel(), _on(slopes, prefix, doc, position)
        rows = {t.shape[0] for t in (prefix, doc, position) if t is not None}
        self.sequences = None if not rows else rows.pop() if len(rows) == 1 else -1        # (-1: they disagree)
        self.columns = min((t.shape[1] for t in (doc, position) if t is not None), default=None)
        strides = {t.stride(0) if t.shape[0] > 1 else t.shape[1] for t in (doc, position) if t is not None}
        if len(strides) > 1:
            raise TypeError("doc and position must have rows of one length")
        self.desc = _Score(_p(slopes), _p(prefix), _p(doc), _p(position), scale, cap, window, strides.pop() if strides else 0)
        self._ref = byref(self.desc)

    def _check(self, batch, q_heads):
        if self.heads is not None and self.heads != q_heads:
            raise ValueError("slopes: one for each query head")
        if self.sequences is not None and self.sequences != batch.sequences:
            raise ValueError("prefix, doc and position: one row for each sequence")
        if self.columns is not None and self.columns < batch.max_len:
            raise ValueError("doc and position: an entry for each of max_len cached tokens")


class Rope:
    """Tables of cosines and sines (positions, pairs), float32; sections: pairs on each axis (default: all on one)."""

    def __init__(self, cos, sin, sections=None, interleaved=False):
        _types()
        self.cos, self.sin = _floats(cos, "cos"), _floats(sin, "sin", cos.shape)
        self.sections = [cos.shape[1]] if sections is None else [int(x) for x in sections]
        if not 1 <= len(self.sections) <= 4:
            raise ValueError("one to four axes")
        self.axes, self._at = len(self.sections), _on(cos, sin)
        self.desc = _Rope(_p(cos), _p(sin), cos.shape[0], cos.shape[1], self.axes, int(interleaved),
                          (c_int32 * 4)(*self.sections))
        self._ref = byref(self.desc)


def _rows(q, cache, batch, what="q"):
    """Query heads and the distance of rows of q: (tokens, q_heads, head_dim), dense but for that distance."""
    batch._fits(cache)
    shape = q.shape
    if len(shape) != 3 or shape[0] != batch.tokens or shape[2] != cache.head_dim or q.dtype is not cache.dtype:
        raise TypeError(f"{what} must be (tokens, q_heads, head_dim) in the cache's type")
    heads, d = shape[1], shape[2]
    apart, across, along = q.stride()
    if (along != 1 or (across != d and heads > 1)) and q.numel():
        raise TypeError(f"heads of {what} must be dense")
    return heads, apart if shape[0] > 1 else heads * d


def _turned(cache, batch, rope, qkv, position, q, cache_position):
    """Query heads, type and distance of rows of qkv, and of cache_position, of a call that rotates."""
    hq, width = _rows(q, cache, batch)
    tokens, d = batch.tokens, cache.head_dim
    if width != hq * d or qkv.shape != (tokens, (hq + 2 * cache.kv_heads) * d):
        raise TypeError("qkv must be (tokens, (q_heads + 2 kv_heads) head_dim), q dense")
    apart, along = qkv.stride()
    if along != 1 and qkv.numel():
        raise TypeError("rows of qkv must be dense")
    if position.dtype is not _i32 or position.shape != (rope.axes, tokens) or not position.is_contiguous():
        raise TypeError("position must be int32, (axes, tokens)")
    if _ints(cache_position, "cache_position", 2) is not None and cache_position.shape[0] != batch.sequences:
        raise ValueError("cache_position: one row for each sequence")
    if cache_position is not None and cache_position.shape[1] < batch.max_len:
        raise ValueError("cache_position: an entry for each of max_len cached tokens")
    stride = 0 if cache_position is None else cache_position.stride(0) if batch.sequences > 1 else cache_position.shape[1]
    return hq, _b._xdtype(qkv), apart if tokens > 1 else qkv.shape[1], stride


def rope_append(cache: KVCache, batch: Batch, rope: Rope, qkv, position, q, weights=None, cache_position=None):
    """qkv: (tokens, (q_heads + 2 kv_heads) head_dim), float32 or bfloat16, dense rows; position: int32 (axes, tokens); q: gets the
    rotated queries (tokens, q_heads, head_dim) in the cache's type.  weights: sums of the new slots, set to zero;
    cache_position: int32 (sequences, at least max_len), gets the positions on axis 0."""
    hq, x, apart, stride = _turned(cache, batch, rope, qkv, position, q, cache_position)
    _ck(load().bwla_rope_append(cache._ref, batch._ref, rope._ref, _p(position), _p(qkv), x, apart, hq,
                                _p(q), _p(cache._of(weights, "weights")), _p(cache_position), stride, _s()), "bwla_rope_append")
    return q


def attention_workspace_size(cache: KVCache, batch: Batch, q_heads: int, weights: bool = False) -> int:
    out = c_size_t()
    _ck(load().bwla_attention_workspace_size(cache._ref, batch._ref, q_heads, int(weights), byref(out)), "bwla_attention_workspace_size")
    return out.value


def attention_forward(cache: KVCache, batch: Batch, score: Score, q, out, lse=None, weights=None, ws=None):
    """out (tokens, q_heads, head_dim, dense) = softmax attention of the new tokens over the cache.  lse: float32 (tokens, q_heads);
    weights: sums that the softmax weights are added to (needs lse); ws: attention_workspace_size bytes."""
    hq, stride = _rows(q, cache, batch)
    if out.shape != q.shape or out.dtype != q.dtype or not out.is_contiguous():
        raise TypeError("out must be like q, and dense")
    score._check(batch, hq)
    _floats(lse, "lse", (batch.tokens, hq))
    _ck(load().bwla_attention_forward(cache._ref, batch._ref, score._ref, _p(q), stride, hq, _p(out), _p(lse), _p(cache._of(weights, "weights")),
                                      _p(ws), _bytes(ws), _s()), "bwla_attention_forward")
    return out


def attention_weights_workspace_size(cache: KVCache, batch: Batch, q_heads: int) -> int:
    out = c_size_t()
    _ck(load().bwla_attention_weights_workspace_size(cache._ref, batch._ref, q_heads, byref(out)), "bwla_attention_weights_workspace_size")
    return out.value


def attention_weights(cache: KVCache, batch: Batch, score: Score, q, lse, weights, ws=None):
    """Adds the softmax weights of these queries, whose lse an attention call left, to the cached tokens' sums."""
    hq, stride = _rows(q, cache, batch)
    score._check(batch, hq)
    _floats(lse, "lse", (batch.tokens, hq))
    _ck(load().bwla_attention_weights(cache._ref, batch._ref, score._ref, _p(q), stride, hq, _p(lse), _p(cache._of(weights, "weights")),
                                      _p(ws), _bytes(ws), _s()), "bwla_attention_weights")
    return weights


def cache_evict_workspace_size(cache: KVCache, batch: Batch) -> int:
    out = c_size_t()
    _ck(load().bwla_cache_evict_workspace_size(cache._ref, batch._ref, byref(out)), "bwla_cache_evict_workspace_size")
    return out.value


def cache_evict(cache: KVCache, batch: Batch, table_out, weights, keep: int, sinks: int, recent: int, length_out, kept=None, position=None,
                position_out=None, ws=None):
    """Each sequence's `keep` heaviest tokens (its first `sinks` and last `recent` among them) to the pages of table_out
    (sequences, pages); length_out gets their number, kept (sequences, keep) their indices, position_out (sequences, keep) their
    entries of position (sequences, at least max_len)."""
    n = batch.sequences
    batch._fits(cache)
    _ints(table_out, "table_out", 2), _ints(length_out, "length_out", 1)
    if table_out.shape[0] != n or length_out.shape[0] != n:
        raise ValueError("table_out and length_out: one row for each sequence")
    if table_out.shape[1] * cache.page_size < min(keep, batch.max_len):
        raise ValueError("table_out: too few pages for keep")
    for t, what in ((kept, "kept"), (position_out, "position_out")):
        if _ints(t, what, 2) is not None and (tuple(t.shape) != (n, keep) or not t.is_contiguous()):
            raise TypeError(f"{what} must be (sequences, keep), dense")
    if _ints(position, "position", 2) is not None and position.shape[0] != n:
        raise ValueError("position: one row for each sequence")
    if position is not None and position.shape[1] < batch.max_len:
        raise ValueError("position: an entry for each of max_len cached tokens")
    if keep == 0:                                      # (an empty tensor has no address)
        position = position_out = None
    row = lambda t: 0 if t is None else t.stride(0) if n > 1 else t.shape[1]  # noqa: E731
    _ck(load().bwla_cache_evict(cache._ref, batch._ref, _p(table_out), row(table_out), _p(cache._of(weights, "weights")), keep, sinks, recent,
                                _p(length_out), _p(kept), _p(position), row(position), _p(position_out), _p(ws), _bytes(ws), _s()),
        "bwla_cache_evict")
    return length_out


# ---------------------------------------------------------------- a cache in 8 bits, normed heads, a step's tables
def _here(at, descriptors, *tensors):
    """The current stream, if what a call is given lies on the current GPU, `at`.  (The library would follow whatever address it gets.)"""
    if at < 0:
        raise TypeError("tensors of this call must lie on a GPU, one for all")
    for d in descriptors:
        if d._at is not None and d._at != at:
            raise ValueError("tensors of this call must lie on one GPU")
    for t in tensors:
        if t is not None and t.get_device() != at:
            raise ValueError("tensors of this call must lie on one GPU")
    stream = _s()
    if at != _b._torch._C._cuda_getDevice():
        raise ValueError("tensors of this call must lie on the current GPU")
    return stream


class KVCache8:
    """Keys and values in pages, a byte each: two tensors (pages, kv_heads, page_size, head_dim) of int8 or float8_e4m3fn, of any strides
    (the same for both) with dense columns, and their scales (pages, kv_heads), float32, rows alike.  dtype: that of queries and
    outputs, bfloat16 or float32."""

    def __init__(self, k, v, k_scale, v_scale, dtype):
        import torch
        _types()
        if k.dim() != 4 or k.shape != v.shape or k.stride() != v.stride() or k.dtype != v.dtype:
            raise TypeError("k and v must be alike: (pages, kv_heads, page_size, head_dim)")
        if k.dtype not in (torch.int8, torch.float8_e4m3fn):
            raise TypeError("codes must be int8 or float8_e4m3fn")
        if k.stride(3) != 1 and k.shape[3] > 1:
            raise TypeError("a head's columns must be dense")
        if dtype not in (torch.bfloat16, torch.float32):
            raise TypeError("dtype must be bfloat16 or float32")
        for t in (k_scale, v_scale):
            if t.dtype is not _f32 or t.shape != k.shape[:2] or t.stride() != k_scale.stride() or (t.shape[1] > 1 and t.stride(1) != 1):
                raise TypeError("scales must be float32, (pages, kv_heads), rows dense and alike")
        self.k, self.v, self.k_scale, self.v_scale, self.dtype, self._at = k, v, k_scale, v_scale, dtype, _on(k, v, k_scale, v_scale)
        self.pages, self.kv_heads, self.page_size, self.head_dim = k.shape
        self.code = CODE_I8 if k.dtype is torch.int8 else CODE_E4M3
        apart = k_scale.stride(0) if self.pages > 1 else self.kv_heads
        self.desc = _Cache8(_p(k), _p(v), _p(k_scale), _p(v_scale), k.stride(0), k.stride(1), k.stride(2), apart, self.pages, self.page_size,
                            self.kv_heads, self.head_dim, self.code, _b.BWLA_X_BF16 if dtype is torch.bfloat16 else _b.BWLA_X_F32)
        self._ref = byref(self.desc)

    @classmethod
    def empty(cls, pages, kv_heads, page_size, head_dim, dtype, code=None, device="cuda"):
        """A cache of its own memory; code: torch.int8 (default) or torch.float8_e4m3fn."""
        import torch
        k, v = (torch.zeros(pages, kv_heads, page_size, head_dim, dtype=torch.int8, device=device).view(code or torch.int8) for _ in range(2))
        return cls(k, v, *(torch.zeros(pages, kv_heads, device=device) for _ in range(2)), dtype)


class HeadNorm:
    """Norms of the query and key heads.  q, k: weights, float32, (head_dim) or one row for each head (heads, head_dim); None: 1."""

    def __init__(self, q=None, k=None, eps=1e-6, centered=False):
        _types()
        for t in (q, k):
            if t is not None and (t.dtype is not _f32 or t.dim() not in (1, 2) or (t.stride(-1) != 1 and t.shape[-1] > 1)):
                raise TypeError("weights must be float32, (head_dim) or (heads, head_dim), dense rows")
        self.q, self.k, self._at = q, k, _on(q, k)
        apart = lambda t: 0 if t is None or t.dim() == 1 else t.stride(0) if t.shape[0] > 1 else t.shape[1]  # noqa: E731
        self.desc = _HeadNorm(_p(q), _p(k), apart(q), apart(k), eps, int(centered))
        self._ref = byref(self.desc)

    def _check(self, cache, q_heads):
        for t, heads in ((self.q, q_heads), (self.k, cache.kv_heads)):
            if t is not None and (t.shape[-1] != cache.head_dim or (t.dim() == 2 and t.shape[0] != heads)):
                raise ValueError("weights: head_dim of them, for all heads or for each")


def norm_rope_append(cache, batch: Batch, rope: Rope, norm, qkv, position, q, weights=None, cache_position=None):
    """rope_append of normed queries and keys (norm: HeadNorm, or None), into a KVCache or a KVCache8 (which has no sums of weights)."""
    hq, x, apart, stride = _turned(cache, batch, rope, qkv, position, q, cache_position)
    if norm is not None:
        norm._check(cache, hq)
    eight = isinstance(cache, KVCache8)
    if eight and weights is not None:
        raise TypeError("a KVCache8 has no sums of weights")
    stream = _here(cache._at, (batch, rope) if norm is None else (batch, rope, norm), qkv, position, q, weights, cache_position)
    args = (cache._ref, batch._ref, rope._ref, None if norm is None else norm._ref, _p(position), _p(qkv), x, apart, hq, _p(q))
    if eight:
        _ck(load().bwla_norm_rope_append8(*args, _p(cache_position), stride, stream), "bwla_norm_rope_append8")
    else:
        _ck(load().bwla_norm_rope_append(*args, _p(cache._of(weights, "weights")), _p(cache_position), stride, stream), "bwla_norm_rope_append")
    return q


def cache8_read(cache: KVCache8, batch: Batch, k=None, v=None):
    """k, v (either may be None): get the values of every sequence's cached tokens, (sequences, max_len, kv_heads, head_dim), float32 or bfloat16,
    dense; 0 behind a sequence's length and in pages that do not exist."""
    batch._fits(cache)
    one = k if k is not None else v
    for t in (k, v):
        if t is not None and (tuple(t.shape) != (batch.sequences, batch.max_len, cache.kv_heads, cache.head_dim) or not t.is_contiguous() or
                              t.dtype is not one.dtype):
            raise TypeError("k and v must be (sequences, max_len, kv_heads, head_dim), dense, of one type")
    if one is None:
        return k, v
    stream = _here(cache._at, (batch,), k, v)
    _ck(load().bwla_cache8_read(cache._ref, batch._ref, _p(k), _p(v), _b._xdtype(one), stream), "bwla_cache8_read")
    return k, v


def attention8_workspace_size(cache: KVCache8, batch: Batch, q_heads: int) -> int:
    out = c_size_t()
    _ck(load().bwla_attention8_workspace_size(cache._ref, batch._ref, q_heads, byref(out)), "bwla_attention8_workspace_size")
    return out.value


def attention8_forward(cache: KVCache8, batch: Batch, score: Score, q, out, lse=None, ws=None):
    """attention_forward over a cache in 8 bits.  ws: attention8_workspace_size bytes."""
    hq, stride = _rows(q, cache, batch)
    if out.shape != q.shape or out.dtype != q.dtype or not out.is_contiguous():
        raise TypeError("out must be like q, and dense")
    score._check(batch, hq)
    _floats(lse, "lse", (batch.tokens, hq))
    stream = _here(cache._at, (batch, score), q, out, lse, ws)
    _ck(load().bwla_attention8_forward(cache._ref, batch._ref, score._ref, _p(q), stride, hq, _p(out), _p(lse), _p(ws), _bytes(ws), stream),
        "bwla_attention8_forward")
    return out


class PagePool:
    """Free pages.  ring (capacity): int32; state (2): int32, the ring's front and how many pages lie there; state_out: where a call
    leaves both (None: in state).  pages: of the pool (default: capacity; where there are more, pages given back that the ring has no room for
    are lost)."""

    def __init__(self, ring, state, page_size, state_out=None, pages=None):
        _types()
        for t, what in ((ring, "ring"), (state, "state"), (state_out, "state_out")):
            if _ints(t, what, 1) is not None and not t.is_contiguous():
                raise TypeError(f"{what} must be dense")
        if state.shape[0] != 2 or (state_out is not None and state_out.shape[0] != 2):
            raise TypeError("state and state_out must have two entries")
        self.ring, self.state, self.state_out, self.page_size = ring, state, state if state_out is None else state_out, int(page_size)
        self._at = _on(ring, state, state_out)
        self.desc = _Pool(_p(ring), _p(state), _p(self.state_out), ring.shape[0] if pages is None else pages, ring.shape[0], self.page_size)
        self._ref = byref(self.desc)

    @classmethod
    def full(cls, pages, page_size, device="cuda"):
        """A pool of which every page is free."""
        import torch
        return cls(torch.arange(pages, dtype=torch.int32, device=device), torch.tensor([0, pages], dtype=torch.int32, device=device), page_size)


def batch_build_workspace_size(sequences: int, tokens: int) -> int:
    out = c_size_t()
    _ck(load().bwla_batch_build_workspace_size(sequences, tokens, byref(out)), "bwla_batch_build_workspace_size")
    return out.value


def _vector(t, what, size):
    if t is not None and (t.dtype is not _i32 or t.shape != (size,) or not t.is_contiguous()):
        raise TypeError(f"{what} must be a dense int32 tensor of {size} entries")


def batch_build(pool: PagePool, table, length, new, length_out, first, status, tokens, max_len, done=None, shift=None, position=None,
                slot=None, sequence=None, ws=None):
    """A step's tables: table (sequences, pages of the longest) gets the pages of the new tokens, length_out (may be length) the lengths,
    first (sequences + 1) the rows; position, slot (int64), sequence (tokens): of each row, or None.  length, new: cached and new tokens
    of each request; done: requests whose place a new one takes; shift: position less index in the cache.  status (4): pages missing,
    requests longer than max_len, rows missing, new tokens; unless the first three are 0 the batch is empty.  All int32 but slot.
    ws: batch_build_workspace_size bytes."""
    n, columns = table.shape
    _vector(length, "length", n), _vector(new, "new", n), _vector(done, "done", n), _vector(shift, "shift", n), _vector(length_out, "length_out", n)
    _vector(first, "first", n + 1), _vector(status, "status", 4), _vector(position, "position", tokens), _vector(sequence, "sequence", tokens)
    _ints(table, "table", 2)
    if slot is not None and (slot.dtype is not _i64 or slot.shape != (tokens,) or not slot.is_contiguous()):
        raise TypeError("slot must be a dense int64 tensor of an entry for each row")
    if columns * pool.page_size < max_len:
        raise ValueError("table: too few pages for max_len")
    stride = table.stride()[0] if n > 1 else columns
    if stride < columns:
        raise TypeError("rows of the table overlap")
    if n == 0:                                         # (an empty tensor has no address)
        length = new = done = shift = table = length_out = None
    if tokens == 0:
        position = slot = sequence = None
    stream = _here(pool._at, (), table, length, new, length_out, first, status, done, shift, position, slot, sequence, ws)
    _ck(load().bwla_batch_build(pool._ref, _p(length), _p(new), _p(done), _p(shift), _p(table), stride, n, tokens, max_len, _p(length_out),
                                _p(first), _p(position), _p(slot), _p(sequence), _p(status), _p(ws), _bytes(ws), stream), "bwla_batch_build")
    return first
