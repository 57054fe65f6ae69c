"""Refusals of the calls around a serving step's attention (normed heads, the cache in 8 bits, a step's tables): checked on the host, nothing
is enqueued (no GPU)."""
import ctypes
import os
from ctypes import byref, c_size_t, c_void_p

import pytest

from paper_2605_00422_amd import attention_binding as A
from paper_2605_00422_amd import binding as B

P = c_void_p(1 << 20)                                  # never followed: every call here is refused, or has nothing to do
OFF = c_void_p((1 << 20) + 8)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2605_00422_amd.build import build_library
        build_library()
    return A.load()


def cache(**kw):
    d = dict(d_k=P, d_v=P, d_k_scale=P, d_v_scale=P, page_stride=8 * 16 * 128, head_stride=16 * 128, slot_stride=128, scale_stride=8, pages=10,
             page_size=16, kv_heads=8, head_dim=128, code=A.CODE_I8, dtype=B.BWLA_X_BF16)
    return A._Cache8(**{**d, **kw})


def plain(**kw):
    d = dict(d_k=P, d_v=P, page_stride=8 * 16 * 128, head_stride=16 * 128, slot_stride=128, pages=10, page_size=16, kv_heads=8, head_dim=128,
             dtype=B.BWLA_X_BF16)
    return A._Cache(**{**d, **kw})


def batch(**kw):
    d = dict(d_table=P, d_len=P, d_first=P, tokens=5, sequences=2, table_stride=4, max_new=3, max_len=60)
    return A._Batch(**{**d, **kw})


def score(**kw):
    return A._Score(**{**dict(scale=0.1), **kw})


def norm(**kw):
    return A._HeadNorm(**{**dict(d_q=P, d_k=P, q_stride=0, k_stride=0, eps=1e-6, centered=0), **kw})


def forward(lib, c=None, b=None, s=None, q=P, stride=16 * 128, hq=16, out=P, lse=P, ws=P, ws_bytes=1 << 40):
    return lib.bwla_attention8_forward(None if c is False else byref(c or cache()), byref(b or batch()), byref(s or score()), q, stride, hq, out, lse, ws,
                                       ws_bytes, None)


def rope(**kw):
    return A._Rope(**{**dict(d_cos=P, d_sin=P, rows=100, pairs=64, axes=1, interleaved=0, sections=(ctypes.c_int32 * 4)(64, 0, 0, 0)), **kw})


def append8(lib, c=None, b=None, n=None, r=None, position=P, qkv=P, xd=0, stride=32 * 128, hq=16, q=P, cpos=None, cstride=0):
    return lib.bwla_norm_rope_append8(byref(c or cache()), byref(b or batch()), byref(r or rope()), None if n is False else byref(n or norm()), position, qkv,
                                      xd, stride, hq, q, cpos, cstride, None)


def append(lib, c=None, b=None, n=None, r=None, position=P, qkv=P, xd=0, stride=32 * 128, hq=16, q=P, weights=None):
    return lib.bwla_norm_rope_append(byref(c or plain()), byref(b or batch()), byref(r or rope()), byref(n or norm()), position, qkv, xd, stride, hq, q,
                                     weights, None, 0, None)


def read(lib, c=None, b=None, k=P, v=P, t=0):
    return lib.bwla_cache8_read(byref(c or cache()), byref(b or batch()), k, v, t, None)


SHAPES = [
    (dict(pages=0), {}, B.BWLA_ERR_SHAPE), (dict(page_size=0), {}, B.BWLA_ERR_SHAPE), (dict(kv_heads=0), {}, B.BWLA_ERR_SHAPE),
    (dict(head_dim=0), {}, B.BWLA_ERR_SHAPE), (dict(head_dim=24), {}, B.BWLA_ERR_UNSUPPORTED), (dict(head_dim=272, slot_stride=272), {}, B.BWLA_ERR_UNSUPPORTED),
    (dict(page_size=24), {}, B.BWLA_ERR_UNSUPPORTED), (dict(page_size=4), {}, B.BWLA_ERR_UNSUPPORTED), (dict(dtype=7), {}, B.BWLA_ERR_UNSUPPORTED),
    (dict(code=2), {}, B.BWLA_ERR_UNSUPPORTED), (dict(code=-1), {}, B.BWLA_ERR_UNSUPPORTED),
    ({}, dict(sequences=-1), B.BWLA_ERR_SHAPE), ({}, dict(tokens=-1), B.BWLA_ERR_SHAPE), ({}, dict(max_len=65), B.BWLA_ERR_SHAPE),
    ({}, dict(max_len=-1), B.BWLA_ERR_SHAPE), ({}, dict(max_len=(1 << 24) + 1, table_stride=1 << 24), B.BWLA_ERR_UNSUPPORTED),
    ({}, dict(sequences=70000), B.BWLA_ERR_UNSUPPORTED),
]
CACHES = [
    (dict(d_k=None), {}, B.BWLA_ERR_NULL), (dict(d_v=None), {}, B.BWLA_ERR_NULL), (dict(d_k=OFF), {}, B.BWLA_ERR_ALIGN),
    (dict(d_k_scale=None), {}, B.BWLA_ERR_NULL), (dict(d_v_scale=None), {}, B.BWLA_ERR_NULL), (dict(d_v_scale=OFF), {}, B.BWLA_ERR_ALIGN),
    (dict(scale_stride=7), {}, B.BWLA_ERR_SHAPE), (dict(page_stride=-16), {}, B.BWLA_ERR_SHAPE), (dict(slot_stride=64), {}, B.BWLA_ERR_SHAPE),
    (dict(slot_stride=136), {}, B.BWLA_ERR_ALIGN), (dict(head_stride=2056), {}, B.BWLA_ERR_ALIGN), (dict(page_stride=16392), {}, B.BWLA_ERR_ALIGN),
    ({}, dict(d_len=None), B.BWLA_ERR_NULL), ({}, dict(d_table=None), B.BWLA_ERR_NULL),
]


@pytest.mark.parametrize("c,b,status", SHAPES + CACHES)
def test_what_every_call_of_the_cache_refuses(lib, c, b, status):
    c, b = cache(**c), batch(**b)
    assert forward(lib, c, b) == status
    assert append8(lib, c, b) == status
    assert read(lib, c, b) == status


@pytest.mark.parametrize("c,b,status", SHAPES)
def test_workspace_size_refuses(lib, c, b, status):
    n = c_size_t(7)
    c, b = cache(**c), batch(**b)
    assert lib.bwla_attention8_workspace_size(byref(c), byref(b), c.kv_heads, byref(n)) == status and n.value == 7


def test_null_descriptors(lib):
    n = c_size_t()
    assert forward(lib, False) == B.BWLA_ERR_NULL
    assert lib.bwla_attention8_workspace_size(None, byref(batch()), 8, byref(n)) == B.BWLA_ERR_NULL
    assert lib.bwla_attention8_workspace_size(byref(cache()), byref(batch()), 8, None) == B.BWLA_ERR_NULL
    assert lib.bwla_attention8_workspace_size(byref(cache()), None, 8, byref(n)) == B.BWLA_ERR_NULL
    assert lib.bwla_cache8_read(None, byref(batch()), P, P, 0, None) == B.BWLA_ERR_NULL
    assert lib.bwla_norm_rope_append8(None, byref(batch()), byref(rope()), None, P, P, 0, 4096, 16, P, None, 0, None) == B.BWLA_ERR_NULL
    assert lib.bwla_norm_rope_append(None, byref(batch()), byref(rope()), None, P, P, 0, 4096, 16, P, None, None, 0, None) == B.BWLA_ERR_NULL
    assert lib.bwla_batch_build(None, P, P, None, None, P, 4, 2, 5, 60, P, P, None, None, None, P, P, 1 << 20, None) == B.BWLA_ERR_NULL


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), B.BWLA_ERR_NULL), (dict(out=None), B.BWLA_ERR_NULL), (dict(q=OFF), B.BWLA_ERR_ALIGN), (dict(out=OFF), B.BWLA_ERR_ALIGN),
    (dict(stride=15 * 128), B.BWLA_ERR_SHAPE), (dict(stride=16 * 128 + 4), B.BWLA_ERR_ALIGN), (dict(hq=12), B.BWLA_ERR_SHAPE), (dict(hq=0), B.BWLA_ERR_SHAPE),
    (dict(s=score(scale=0.0)), B.BWLA_ERR_SHAPE), (dict(s=score(scale=float("nan"))), B.BWLA_ERR_SHAPE), (dict(s=score(cap=-1.0)), B.BWLA_ERR_SHAPE),
    (dict(s=score(window=-1)), B.BWLA_ERR_SHAPE), (dict(s=score(scale=8e-39)), B.BWLA_ERR_UNSUPPORTED), (dict(s=score(d_doc=P, index_stride=59)), B.BWLA_ERR_SHAPE),
    (dict(b=batch(max_len=60, sequences=2, table_stride=400, max_new=1, d_first=None, tokens=2), ws=None), B.BWLA_OK),
    (dict(b=batch(max_len=6400, table_stride=400), ws=None), B.BWLA_ERR_NULL), (dict(b=batch(max_len=6400, table_stride=400), ws_bytes=16), B.BWLA_ERR_BUFSIZE),
    (dict(b=batch(max_len=6400, table_stride=400), ws=OFF), B.BWLA_ERR_ALIGN), (dict(b=batch(d_first=None)), B.BWLA_ERR_SHAPE)])
def test_attention8_refuses(lib, kw, status):
    # (8e-39 log2(e) = 1.154e-38 lies below 2^-126 = 1.175e-38, the least normal number; 1e-38 log2(e) does not)
    if status == B.BWLA_OK:                            # (nothing is called that would run: the workspace alone is asked for)
        n = c_size_t(7)
        assert lib.bwla_attention8_workspace_size(byref(cache()), byref(kw["b"]), 16, byref(n)) == B.BWLA_OK and n.value == 0
        return
    assert forward(lib, **kw) == status


@pytest.mark.parametrize("n,status", [
    (dict(eps=0.0), B.BWLA_ERR_SHAPE), (dict(eps=-1e-6), B.BWLA_ERR_SHAPE), (dict(eps=float("nan")), B.BWLA_ERR_SHAPE), (dict(eps=float("inf")), B.BWLA_ERR_SHAPE),
    (dict(eps=1e-44), B.BWLA_ERR_SHAPE), (dict(d_q=OFF), B.BWLA_ERR_ALIGN), (dict(d_k=OFF), B.BWLA_ERR_ALIGN), (dict(q_stride=64), B.BWLA_ERR_SHAPE),
    (dict(k_stride=-128), B.BWLA_ERR_SHAPE), (dict(q_stride=130), B.BWLA_ERR_ALIGN)])
def test_norms_refused(lib, n, status):
    assert append8(lib, n=norm(**n)) == status and append(lib, n=norm(**n)) == status


@pytest.mark.parametrize("kw,status", [
    (dict(qkv=None), B.BWLA_ERR_NULL), (dict(q=None), B.BWLA_ERR_NULL), (dict(position=None), B.BWLA_ERR_NULL), (dict(qkv=OFF), B.BWLA_ERR_ALIGN),
    (dict(stride=32 * 128 - 1), B.BWLA_ERR_SHAPE), (dict(stride=32 * 128 + 2), B.BWLA_ERR_ALIGN), (dict(xd=5), B.BWLA_ERR_UNSUPPORTED),
    (dict(r=rope(pairs=65)), B.BWLA_ERR_SHAPE), (dict(r=rope(axes=5)), B.BWLA_ERR_SHAPE), (dict(r=rope(rows=0)), B.BWLA_ERR_SHAPE),
    (dict(r=rope(d_cos=None)), B.BWLA_ERR_NULL)])
def test_appends_refuse(lib, kw, status):
    assert append8(lib, **kw) == status and append(lib, **kw) == status


def test_positions_of_the_cache_need_room(lib):
    assert append8(lib, cpos=P, cstride=59) == B.BWLA_ERR_SHAPE


def test_read_refuses_and_has_nothing_to_do(lib):
    assert read(lib, t=3) == B.BWLA_ERR_UNSUPPORTED and read(lib, k=OFF) == B.BWLA_ERR_ALIGN
    assert read(lib, k=None, v=None) == B.BWLA_OK and read(lib, b=batch(sequences=0)) == B.BWLA_OK
    assert read(lib, b=batch(max_len=0)) == B.BWLA_OK


def test_calls_without_rows_do_nothing(lib):
    for b in (batch(tokens=0), batch(sequences=0), batch(max_new=0)):
        assert forward(lib, b=b) == B.BWLA_OK
    for b in (batch(tokens=0), batch(sequences=0)):
        assert append8(lib, b=b) == B.BWLA_OK and append(lib, b=b) == B.BWLA_OK


def pool(**kw):
    return A._Pool(**{**dict(d_ring=P, d_state=P, d_state_out=P, pages=10, capacity=10, page_size=16), **kw})


def build(lib, p=None, length=P, new=P, done=None, shift=None, table=P, stride=4, sequences=2, tokens=5, max_len=60, length_out=P, first=P, status=P, ws=P,
          ws_bytes=1 << 20):
    return lib.bwla_batch_build(byref(p or pool()), length, new, done, shift, table, stride, sequences, tokens, max_len, length_out, first, None, None, None,
                                status, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(p=pool(capacity=0)), B.BWLA_ERR_SHAPE), (dict(p=pool(pages=0)), B.BWLA_ERR_SHAPE), (dict(p=pool(page_size=0)), B.BWLA_ERR_SHAPE),
    (dict(p=pool(page_size=12)), B.BWLA_ERR_UNSUPPORTED), (dict(p=pool(page_size=1 << 17)), B.BWLA_ERR_UNSUPPORTED), (dict(p=pool(pages=1 << 31)), B.BWLA_ERR_UNSUPPORTED),
    (dict(p=pool(d_ring=None)), B.BWLA_ERR_NULL), (dict(p=pool(d_state=None)), B.BWLA_ERR_NULL), (dict(p=pool(d_state_out=None)), B.BWLA_ERR_NULL),
    (dict(length=None), B.BWLA_ERR_NULL), (dict(new=None), B.BWLA_ERR_NULL), (dict(table=None), B.BWLA_ERR_NULL), (dict(length_out=None), B.BWLA_ERR_NULL),
    (dict(first=None), B.BWLA_ERR_NULL), (dict(status=None), B.BWLA_ERR_NULL), (dict(ws=None), B.BWLA_ERR_NULL), (dict(ws=OFF), B.BWLA_ERR_ALIGN),
    (dict(ws_bytes=16), B.BWLA_ERR_BUFSIZE), (dict(sequences=-1), B.BWLA_ERR_SHAPE), (dict(tokens=-1), B.BWLA_ERR_SHAPE), (dict(max_len=-1), B.BWLA_ERR_SHAPE),
    (dict(max_len=65), B.BWLA_ERR_SHAPE), (dict(sequences=70000), B.BWLA_ERR_UNSUPPORTED), (dict(tokens=1 << 24), B.BWLA_ERR_UNSUPPORTED),
    (dict(max_len=(1 << 24) + 1, stride=1 << 24), B.BWLA_ERR_UNSUPPORTED)])
def test_build_refuses(lib, kw, status):
    assert build(lib, **kw) == status


def test_build_workspace_size(lib):
    n = c_size_t(7)
    assert lib.bwla_batch_build_workspace_size(-1, 5, byref(n)) == B.BWLA_ERR_SHAPE and lib.bwla_batch_build_workspace_size(1, -5, byref(n)) == B.BWLA_ERR_SHAPE
    assert lib.bwla_batch_build_workspace_size(70000, 5, byref(n)) == B.BWLA_ERR_UNSUPPORTED and lib.bwla_batch_build_workspace_size(1, 5, None) == B.BWLA_ERR_NULL
    assert n.value == 7
    assert A.batch_build_workspace_size(0, 0) >= 16 and A.batch_build_workspace_size(65535, 1 << 20) >= 65535 * 8


# ---------------------------------------------------------------- the binding's own checks, on CPU tensors
torch = pytest.importorskip("torch")


def i32(*s):
    return torch.zeros(*s, dtype=torch.int32)


def codes(pages=6, hkv=2, page=16, d=32, t=torch.int8):
    return [torch.zeros(pages, hkv, page, d, dtype=torch.int8).view(t) for _ in range(2)], [torch.zeros(pages, hkv) for _ in range(2)]


def test_cache8_checks():
    (k, v), (ks, vs) = codes()
    A.KVCache8(k, v, ks, vs, torch.bfloat16)
    for bad in ((k, v[:5], ks, vs, torch.bfloat16), (k.float(), v.float(), ks, vs, torch.bfloat16), (k, v.view(torch.float8_e4m3fn), ks, vs, torch.bfloat16),
                (k, v, ks[:, :1], vs[:, :1], torch.bfloat16), (k, v, ks.double(), vs, torch.bfloat16), (k, v, ks, vs, torch.float16),
                (k.view(torch.float8_e5m2), v.view(torch.float8_e5m2), ks, vs, torch.bfloat16), (k[..., ::2], v[..., ::2], ks, vs, torch.bfloat16),
                (k, v, ks.T.contiguous().T, vs.T.contiguous().T, torch.bfloat16)):
        with pytest.raises(TypeError):
            A.KVCache8(*bad)


def test_tensors_that_are_not_on_a_gpu_are_refused(lib):
    (k, v), (ks, vs) = codes(t=torch.float8_e4m3fn)
    cache8, b = A.KVCache8(k, v, ks, vs, torch.float32), A.Batch(i32(1, 3), i32(1), max_len=40)
    rope_, q, qkv = A.Rope(torch.zeros(4, 16), torch.zeros(4, 16)), torch.zeros(1, 4, 32), torch.zeros(1, 8 * 32)
    with pytest.raises(TypeError, match="GPU"):
        A.attention8_forward(cache8, b, A.Score(1.0), q, torch.zeros_like(q))
    with pytest.raises(TypeError, match="GPU"):
        A.norm_rope_append(cache8, b, rope_, A.HeadNorm(), qkv, i32(1, 1), q)
    with pytest.raises(TypeError, match="GPU"):
        A.cache8_read(cache8, b, torch.zeros(1, 40, 2, 32))
    with pytest.raises(TypeError, match="GPU"):
        A.batch_build(A.PagePool(i32(5), i32(2), 16), i32(1, 3), i32(1), i32(1), i32(1), i32(2), i32(4), 3, 40)
    with pytest.raises(TypeError, match="sums"):
        A.norm_rope_append(cache8, b, rope_, None, qkv, i32(1, 1), q, weights=torch.zeros(6, 2, 16))


def test_norm_and_shape_checks(lib):
    (k, v), (ks, vs) = codes()
    cache8, b = A.KVCache8(k, v, ks, vs, torch.bfloat16), A.Batch(i32(1, 3), i32(1), max_len=40)
    rope_, q, qkv = A.Rope(torch.zeros(4, 16), torch.zeros(4, 16)), torch.zeros(1, 4, 32, dtype=torch.bfloat16), torch.zeros(1, 8 * 32)
    for w in (torch.zeros(31), torch.zeros(3, 32), torch.zeros(5, 32)):
        with pytest.raises(ValueError):
            A.norm_rope_append(cache8, b, rope_, A.HeadNorm(q=w), qkv, i32(1, 1), q)
    for w in (torch.zeros(32, dtype=torch.bfloat16), torch.zeros(1, 4, 32), torch.zeros(64)[::2]):
        with pytest.raises(TypeError):
            A.HeadNorm(k=w)
    with pytest.raises(TypeError):
        A.norm_rope_append(cache8, b, rope_, None, qkv, i32(2, 1), q)
    with pytest.raises(TypeError):
        A.attention8_forward(cache8, b, A.Score(1.0), q, torch.zeros(1, 4, 32))
    with pytest.raises(TypeError):
        A.attention8_forward(cache8, b, A.Score(1.0), q.float(), q.float())
    for t in (torch.zeros(1, 39, 2, 32), torch.zeros(1, 40, 2, 32).transpose(1, 2).contiguous().transpose(1, 2)):
        with pytest.raises(TypeError):
            A.cache8_read(cache8, b, t)
    with pytest.raises(TypeError):
        A.cache8_read(cache8, b, torch.zeros(1, 40, 2, 32), torch.zeros(1, 40, 2, 32, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        A.cache8_read(cache8, A.Batch(i32(1, 2), i32(1), max_len=40), torch.zeros(1, 40, 2, 32))
    assert A.cache8_read(cache8, b) == (None, None)


def test_build_checks(lib):
    pool_ = A.PagePool(i32(5), i32(2), 16)
    good = dict(table=i32(2, 3), length=i32(2), new=i32(2), length_out=i32(2), first=i32(3), status=i32(4), tokens=6, max_len=48)
    for bad in (dict(new=i32(3)), dict(length_out=i32(1)), dict(first=i32(2)), dict(status=i32(3)), dict(position=i32(5)), dict(done=i32(1)),
                dict(table=i32(3, 3)), dict(max_len=49), dict(shift=i32(4)), dict(new=i32(4)[::2])):
        with pytest.raises((ValueError, TypeError)) as e:
            A.batch_build(pool_, **{**good, **bad})
        assert "GPU" not in str(e.value)
    for bad in (dict(slot=i32(6)), dict(slot=torch.zeros(5, dtype=torch.int64)), dict(length=i32(2).long()), dict(table=i32(3).expand(2, 3))):
        with pytest.raises(TypeError) as e:
            A.batch_build(pool_, **{**good, **bad})
        assert "GPU" not in str(e.value)
    for bad in ((i32(5), i32(3), 16), (i32(5).long(), i32(2), 16), (i32(10)[::2], i32(2), 16), (i32(5), i32(2), 16, i32(1))):
        with pytest.raises(TypeError):
            A.PagePool(*bad)
