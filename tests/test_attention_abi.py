"""Refusals of the cache, attention, rotation and eviction calls: checked on the host, nothing is enqueued (no GPU)."""
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
    d = dict(d_k=P, d_v=P, page_stride=8 * 16 * 128, head_stride=16 * 128, slot_stride=128, pages=10, page_size=16, kv_heads=8,
             head_dim=128, dtype=B.BWLA_X_BF16)
    return A._Cache(**{**d, **kw})


def batch(**kw):
    d = dict(d_table=P, d_len=P, d_first=P, tokens=5, sequences=2, table_stride=4, max_new=3, max_len=60)
    return A._Batch(**{**d, **kw})


def score(**kw):
    return A._Score(**{**dict(scale=0.1), **kw})


SHAPES = [  # what every call refuses of a cache and a batch
    (dict(pages=0), {}, B.BWLA_ERR_SHAPE), (dict(page_size=0), {}, B.BWLA_ERR_SHAPE), (dict(kv_heads=0), {}, B.BWLA_ERR_SHAPE),
    (dict(head_dim=0), {}, B.BWLA_ERR_SHAPE), (dict(head_dim=12), {}, B.BWLA_ERR_UNSUPPORTED), (dict(head_dim=264, slot_stride=264), {}, B.BWLA_ERR_UNSUPPORTED),
    (dict(page_size=24), {}, B.BWLA_ERR_UNSUPPORTED), (dict(page_size=4), {}, B.BWLA_ERR_UNSUPPORTED), (dict(dtype=7), {}, B.BWLA_ERR_UNSUPPORTED),
    ({}, dict(sequences=-1), B.BWLA_ERR_SHAPE), ({}, dict(tokens=-1), B.BWLA_ERR_SHAPE), ({}, dict(max_len=65), B.BWLA_ERR_SHAPE),
    ({}, dict(max_len=-1), B.BWLA_ERR_SHAPE), ({}, dict(max_new=-1), B.BWLA_ERR_SHAPE),
    ({}, dict(max_len=(1 << 24) + 1, table_stride=1 << 24), B.BWLA_ERR_UNSUPPORTED), ({}, dict(sequences=70000), B.BWLA_ERR_UNSUPPORTED),
]
CACHES = [  # ... of the pointers and strides
    (dict(d_k=None), {}, B.BWLA_ERR_NULL), (dict(d_v=None), {}, B.BWLA_ERR_NULL), (dict(d_k=OFF), {}, B.BWLA_ERR_ALIGN),
    (dict(page_stride=-16), {}, B.BWLA_ERR_SHAPE), (dict(slot_stride=64), {}, B.BWLA_ERR_SHAPE), (dict(slot_stride=132), {}, B.BWLA_ERR_ALIGN),
    (dict(head_stride=2044), {}, B.BWLA_ERR_ALIGN), (dict(page_stride=16388), {}, B.BWLA_ERR_ALIGN),
    ({}, dict(d_len=None), B.BWLA_ERR_NULL), ({}, dict(d_table=None), B.BWLA_ERR_NULL),
]


def forward(lib, c=None, b=None, s=None, q=P, stride=16 * 128, hq=16, out=P, lse=P, weights=None, ws=P, ws_bytes=1 << 40):
    ref = lambda x: None if x is False else byref(x)  # noqa: E731
    return lib.bwla_attention_forward(ref(cache() if c is None else c), ref(batch() if b is None else b), ref(score() if s is None else s),
                                      q, stride, hq, out, lse, weights, ws, ws_bytes, None)


def evict(lib, c=None, b=None, table=P, stride=4, weights=P, keep=20, sinks=2, recent=3, length=P, kept=P, pos=None, pos_stride=0,
          pos_out=None, ws=P, ws_bytes=1 << 40):
    return lib.bwla_cache_evict(byref(c or cache()), byref(b or batch()), table, stride, weights, keep, sinks, recent, length, kept, pos,
                                pos_stride, pos_out, ws, ws_bytes, None)


def append(lib, c=None, b=None, position=P, qkv=P, xd=0, stride=32 * 128, hq=16, q=P, weights=None, cpos=None, cstride=0, **kw):
    d = dict(d_cos=P, d_sin=P, rows=100, pairs=64, axes=1, interleaved=0, sections=(ctypes.c_int32 * 4)(64, 0, 0, 0))
    return lib.bwla_rope_append(byref(c or cache()), byref(b or batch()), byref(A._Rope(**{**d, **kw})), position, qkv, xd, stride, hq, q,
                                weights, cpos, cstride, None)


@pytest.mark.parametrize("c,b,status", SHAPES + CACHES)
def test_what_every_call_refuses(lib, c, b, status):
    c, b = cache(**c), batch(**b)
    assert forward(lib, c, b) == status
    assert append(lib, c, b) == status
    assert evict(lib, c, b) == status
    assert lib.bwla_attention_weights(byref(c), byref(b), byref(score()), P, 16 * 128, 16, P, P, P, 1 << 40, None) == status


@pytest.mark.parametrize("c,b,status", SHAPES)
def test_sizes_refuse_shapes(lib, c, b, status):
    c, b, n = cache(**c), batch(**b), c_size_t()
    assert lib.bwla_attention_workspace_size(byref(c), byref(b), 16, 0, byref(n)) == status
    assert lib.bwla_attention_weights_workspace_size(byref(c), byref(b), 16, byref(n)) == status
    assert lib.bwla_cache_evict_workspace_size(byref(c), byref(b), byref(n)) == status
    assert lib.bwla_attention_workspace_size(byref(cache()), byref(batch()), 16, 0, None) == B.BWLA_ERR_NULL
    assert lib.bwla_attention_workspace_size(None, byref(batch()), 16, 0, byref(n)) == B.BWLA_ERR_NULL
    assert lib.bwla_cache_evict_workspace_size(None, byref(batch()), byref(n)) == B.BWLA_ERR_NULL


def test_attention_refuses(lib):
    R = B
    assert forward(lib, s=False) == R.BWLA_ERR_NULL
    for bad in (dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=0.1, cap=-1.0),
                dict(scale=0.1, cap=float("nan")), dict(scale=0.1, window=-1), dict(scale=0.1, d_doc=P, index_stride=59),
                dict(scale=0.1, d_position=P, index_stride=59)):
        assert forward(lib, s=A._Score(**bad)) == R.BWLA_ERR_SHAPE, bad
    assert forward(lib, hq=12, stride=12 * 128) == R.BWLA_ERR_SHAPE          # no multiple of the key-value heads
    assert forward(lib, hq=2048, stride=2048 * 128) == R.BWLA_ERR_UNSUPPORTED
    assert forward(lib, stride=16 * 128 - 8) == R.BWLA_ERR_SHAPE
    assert forward(lib, stride=16 * 128 + 4) == R.BWLA_ERR_ALIGN
    assert forward(lib, q=OFF) == R.BWLA_ERR_ALIGN and forward(lib, out=OFF) == R.BWLA_ERR_ALIGN
    assert forward(lib, q=None) == R.BWLA_ERR_NULL and forward(lib, out=None) == R.BWLA_ERR_NULL
    assert forward(lib, weights=P, lse=None) == R.BWLA_ERR_NULL
    assert forward(lib, b=batch(d_first=None)) == R.BWLA_ERR_SHAPE            # five rows of two sequences
    n = c_size_t()
    long = dict(c=cache(pages=1000), b=batch(table_stride=600, max_len=9000))
    assert lib.bwla_attention_workspace_size(byref(long["c"]), byref(long["b"]), 16, 1, byref(n)) == 0 and n.value > 0
    assert forward(lib, **long, weights=P, ws_bytes=n.value - 1) == R.BWLA_ERR_BUFSIZE
    assert forward(lib, **long, weights=P, ws=None) == R.BWLA_ERR_NULL
    assert forward(lib, **long, weights=P, ws=OFF) == R.BWLA_ERR_ALIGN
    w = lambda **k: lib.bwla_attention_weights(byref(cache()), byref(batch()), byref(score()), P, 16 * 128, 16, k.get("lse", P),  # noqa: E731
                                               k.get("weights", P), P, 1 << 40, None)
    assert w(lse=None) == R.BWLA_ERR_NULL and w(weights=None) == R.BWLA_ERR_NULL and w(weights=OFF) == R.BWLA_ERR_ALIGN


def test_rotation_refuses(lib):
    sec = lambda *v: (ctypes.c_int32 * 4)(*v)  # noqa: E731
    assert append(lib, pairs=65, sections=sec(65)) == B.BWLA_ERR_SHAPE
    assert append(lib, sections=sec(63)) == B.BWLA_ERR_SHAPE
    assert append(lib, axes=2, sections=sec(65, -1)) == B.BWLA_ERR_SHAPE
    assert append(lib, axes=0) == B.BWLA_ERR_SHAPE and append(lib, axes=5) == B.BWLA_ERR_SHAPE and append(lib, rows=0) == B.BWLA_ERR_SHAPE
    assert append(lib, stride=32 * 128 - 4) == B.BWLA_ERR_SHAPE and append(lib, stride=32 * 128 + 2) == B.BWLA_ERR_ALIGN
    assert append(lib, xd=5) == B.BWLA_ERR_UNSUPPORTED
    assert append(lib, cpos=P, cstride=59) == B.BWLA_ERR_SHAPE
    for k in ("qkv", "q", "position"):
        assert append(lib, **{k: None}) == B.BWLA_ERR_NULL, k
    assert append(lib, d_cos=None) == B.BWLA_ERR_NULL and append(lib, d_sin=OFF) == B.BWLA_ERR_ALIGN
    assert append(lib, qkv=OFF) == B.BWLA_ERR_ALIGN and append(lib, weights=OFF) == B.BWLA_ERR_ALIGN


def test_eviction_refuses(lib):
    assert evict(lib, keep=-1) == B.BWLA_ERR_SHAPE and evict(lib, keep=4, sinks=2, recent=3) == B.BWLA_ERR_SHAPE
    assert evict(lib, sinks=-1) == B.BWLA_ERR_SHAPE and evict(lib, keep=59, stride=3) == B.BWLA_ERR_SHAPE
    assert evict(lib, pos=P, pos_stride=60) == B.BWLA_ERR_NULL and evict(lib, pos=P, pos_out=P, pos_stride=59) == B.BWLA_ERR_SHAPE
    assert evict(lib, table=None) == B.BWLA_ERR_NULL and evict(lib, length=None) == B.BWLA_ERR_NULL and evict(lib, weights=None) == B.BWLA_ERR_NULL
    assert evict(lib, weights=OFF) == B.BWLA_ERR_ALIGN
    n = c_size_t()
    assert lib.bwla_cache_evict_workspace_size(byref(cache()), byref(batch()), byref(n)) == 0
    assert evict(lib, ws_bytes=n.value - 1) == B.BWLA_ERR_BUFSIZE and evict(lib, ws=None) == B.BWLA_ERR_NULL


def test_nothing_to_do_is_no_error(lib):
    none = batch(sequences=0, tokens=0, d_table=None, d_len=None, d_first=None)
    assert forward(lib, b=none, q=None, out=None) == B.BWLA_OK
    assert append(lib, b=none, qkv=None, q=None) == B.BWLA_OK and evict(lib, b=none) == B.BWLA_OK


def test_binding_refuses_wrong_tensors():
    import torch
    k = torch.zeros(4, 2, 16, 64)
    with pytest.raises(TypeError):
        A.KVCache(k, k.to(torch.bfloat16))
    with pytest.raises(TypeError):
        A.KVCache(k.transpose(2, 3), k.transpose(2, 3))
    with pytest.raises(TypeError):
        A.KVCache(k.half(), k.half())
    c = A.KVCache(k, k.clone())
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(TypeError):
        A.Batch(torch.zeros(2, 4), i(2), max_len=9)
    with pytest.raises(ValueError):
        A.Batch(i(2, 4), i(3), max_len=9)
    with pytest.raises(ValueError):
        A.Batch(i(2, 4), i(2), first=i(3), max_len=9)
    with pytest.raises(ValueError):
        A.Batch(i(2, 4), i(2))
    b = A.Batch(i(2, 4), i(2), max_len=60)
    q = torch.zeros(2, 4, 64)
    for bad in (torch.zeros(3, 4, 64), torch.zeros(2, 4, 32), q.to(torch.bfloat16)):
        with pytest.raises(TypeError):
            A.attention_forward(c, b, A.Score(0.1), bad, bad)
    with pytest.raises(TypeError):
        A.attention_forward(c, b, A.Score(0.1), q, torch.zeros(2, 4, 64, dtype=torch.bfloat16))
    with pytest.raises(TypeError):
        A.attention_forward(c, b, A.Score(0.1), q, q.clone(), lse=torch.zeros(2, 5))
    with pytest.raises(ValueError):
        A.attention_forward(c, b, A.Score(0.1, slopes=torch.zeros(3)), q, q.clone())
    with pytest.raises(ValueError):
        A.attention_forward(c, b, A.Score(0.1, prefix=i(3)), q, q.clone())
    with pytest.raises(TypeError):
        A.Score(0.1, doc=i(2, 8), position=i(2, 9))
    with pytest.raises(ValueError):
        A.Rope(torch.zeros(9, 5), torch.zeros(9, 5), [1] * 5)
    with pytest.raises(TypeError):
        A.rope_append(c, b, A.Rope(torch.zeros(9, 32), torch.zeros(9, 32)), torch.zeros(2, 8 * 64 + 1), i(1, 2), q)
    with pytest.raises(TypeError):
        A.cache_evict(c, b, i(2, 4), c.weights(), 8, 0, 0, i(2), kept=i(2, 9))


def test_sizes_that_do_not_fit_the_kernels_counts(lib):
    out = A.c_size_t()
    size = lambda b, c=None, hq=16: lib.bwla_attention_workspace_size(A.byref(c or cache()), A.byref(b), hq, 0, A.byref(out))  # noqa: E731
    assert size(batch(tokens=(1 << 24) - 1)) == B.BWLA_OK
    assert size(batch(tokens=1 << 24)) == B.BWLA_ERR_UNSUPPORTED
    many = dict(tokens=(1 << 24) - 1, max_new=(1 << 24) - 1)
    assert size(batch(**many)) == B.BWLA_OK
    assert size(batch(**many), cache(kv_heads=1), 1024) == B.BWLA_ERR_UNSUPPORTED      # 2^34 rows
    assert size(batch(tokens=5, max_new=(1 << 24) - 1), cache(kv_heads=1), 1024) == B.BWLA_OK


def test_batch_of_rows_asks_for_its_bounds():
    """One new token each needs neither; with `first` a bound of 1 would leave out all but a sequence's first row."""
    import torch
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    assert A.Batch(i(2, 4), i(2), max_len=9).desc.max_new == 1
    with pytest.raises(ValueError):
        A.Batch(i(2, 4), i(2), first=i(3), tokens=5, max_len=9)
    assert A.Batch(i(2, 4), i(2), first=i(3), tokens=5, max_new=3, max_len=9).desc.max_new == 3


# What the library calls of the runtime to launch, in front of the real one: launches fail on demand, and none reaches a GPU.
FAILING_LAUNCHES = """
static int launches, failing, last;
void fail_at(int n) { launches = 0; failing = n; last = 0; }
int launched(void) { return launches; }
int __hipPushCallConfiguration(void) { return 0; }
int __hipPopCallConfiguration(void) { return 0; }
int hipLaunchKernel(void) { return last = ++launches == failing ? 1 : last; }
int hipGetLastError(void) { int e = last; last = 0; return e; }
int hipPeekAtLastError(void) { return last; }
int hipFuncSetAttribute(void) { return 0; }
int hipGetDevice(int *d) { return *d = 0; }
"""
EACH_LAUNCH = """
import ctypes, sys
sys.path[:0] = [{root!r}, {tests!r}]
hip = ctypes.CDLL({stub!r}, ctypes.RTLD_GLOBAL)         # (in front of the library, which finds its functions first)
import test_attention_abi as t
from paper_2605_00422_amd import binding as B
lib = t.A.load()
hip.fail_at(0)
assert lib.bwla_probe_empty_launch(None) == B.BWLA_OK and hip.launched() == 1, "launches go past the functions above"
long, many = dict(c=t.cache(pages=1000), b=t.batch(table_stride=600, max_len=9000)), t.batch(tokens=90, max_new=60, table_stride=600, max_len=9000)
calls = {{
    "few rows": (1, lambda: t.forward(lib)), "sums": (2, lambda: t.forward(lib, weights=t.P)),
    "parts": (2, lambda: t.forward(lib, **long)), "parts, sums": (3, lambda: t.forward(lib, **long, weights=t.P)),
    "many rows": (1, lambda: t.forward(lib, b=t.batch(tokens=90, max_new=60))),
    "many rows, parts, sums": (3, lambda: t.forward(lib, long["c"], many, weights=t.P)),
    "rotation": (1, lambda: t.append(lib)), "eviction": (2, lambda: t.evict(lib)), "long eviction": (3, lambda: t.evict(lib, **long)),
}}
for name, (least, call) in calls.items():
    hip.fail_at(0)
    status, n = call(), hip.launched()
    assert status == B.BWLA_OK and n >= least, (name, status, n)
    for k in range(1, n + 1):
        hip.fail_at(k)
        status = call()
        assert status == B.BWLA_ERR_HIP, (name, "launch", k, "of", n, "failed", status)
        assert hip.hipGetLastError() == 0, (name, "leaves its error behind")
        assert hip.launched() == k, (name, "goes on after launch", k)
"""


def test_each_launch_that_fails_is_an_error(lib, tmp_path):
    import shutil
    import subprocess
    import sys
    if not shutil.which("gcc"):
        pytest.skip("gcc not available")
    here, stub = os.path.dirname(os.path.abspath(__file__)), str(tmp_path / "hip_failing.so")
    (tmp_path / "hip_failing.c").write_text(FAILING_LAUNCHES)
    subprocess.run(["gcc", "-w", "-shared", "-fPIC", "-o", stub, str(tmp_path / "hip_failing.c")], check=True)
    run = subprocess.run([sys.executable, "-c", EACH_LAUNCH.format(root=os.path.dirname(here), tests=here, stub=stub)], capture_output=True,
                         text=True, timeout=100)
    assert run.returncode == 0, run.stdout + run.stderr


def test_binding_refuses_views_that_are_too_narrow():
    """Views of wide tensors, whose rows lie far enough apart but do not hold what max_len or keep asks for."""
    import torch
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    c = A.KVCache(torch.zeros(4, 2, 16, 64), torch.zeros(4, 2, 16, 64))
    good, narrow = A.Batch(i(2, 9)[:, :4], i(2), max_len=64), A.Batch(i(2, 9)[:, :3], i(2), max_len=49)
    q, wide, short, rope = torch.zeros(2, 4, 64), i(2, 99), i(2, 99)[:, -63:], A.Rope(torch.zeros(9, 32), torch.zeros(9, 32))
    qkv, pos, lse, w = torch.zeros(2, 8 * 64), i(1, 2), torch.zeros(2, 4), c.weights()
    for call in (lambda: A.attention_forward(c, narrow, A.Score(0.1), q, q.clone()),
                 lambda: A.attention_forward(c, good, A.Score(0.1, doc=short), q, q.clone()),
                 lambda: A.attention_forward(c, good, A.Score(0.1, position=short), q, q.clone()),
                 lambda: A.attention_forward(c, good, A.Score(0.1, position=wide, doc=i(2, 99)[:, :63]), q, q.clone()),
                 lambda: A.attention_weights(c, narrow, A.Score(0.1), q, lse, w),
                 lambda: A.attention_weights(c, good, A.Score(0.1, doc=short), q, lse, w),
                 lambda: A.rope_append(c, narrow, rope, qkv, pos, q),
                 lambda: A.rope_append(c, good, rope, qkv, pos, q, w, short),
                 lambda: A.cache_evict(c, narrow, i(2, 4), w, 8, 0, 0, i(2)),
                 lambda: A.cache_evict(c, good, i(2, 9)[:, :2], w, 33, 0, 0, i(2)),
                 lambda: A.cache_evict(c, good, i(2, 4), w, 8, 0, 0, i(2), position=short, position_out=i(2, 8))):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("max_len", [60, 3000])
@pytest.mark.parametrize("ws_bytes", [0, 1 << 40])
def test_eviction_of_all_needs_its_scratch_as_well(lib, max_len, ws_bytes):
    """Integers of the weights are made of long sequences whatever is kept of them."""
    assert evict(lib, b=batch(table_stride=200, max_len=max_len), keep=0, sinks=0, recent=0, ws=None, ws_bytes=ws_bytes) == B.BWLA_ERR_NULL


def test_scales_and_caps_that_fp32_does_not_hold(lib):
    """In base 2 they, or their ratio, are infinite or have lost bits: a cap of 1e-39 makes 0 * inf of a product of 0."""
    for kw in (dict(scale=3e38), dict(scale=1e-40), dict(scale=0.1, cap=3e38), dict(scale=0.1, cap=1e-40), dict(scale=1e4, cap=1e-37), dict(scale=1e-4, cap=1e36)):
        s = score(**kw)
        assert forward(lib, s=s) == B.BWLA_ERR_UNSUPPORTED, kw
        assert lib.bwla_attention_weights(byref(cache()), byref(batch()), byref(s), P, 16 * 128, 16, P, P, P, 1 << 40, None) == B.BWLA_ERR_UNSUPPORTED
    none = batch(sequences=0, tokens=0, d_table=None, d_len=None, d_first=None)
    for kw in (dict(scale=0.1, cap=1e30), dict(scale=1e-6, cap=1e-6), dict(scale=1e6)):
        assert forward(lib, b=none, s=score(**kw), q=None, out=None) == B.BWLA_OK, kw


def test_a_single_element_has_no_stride():
    """One sequence, one page: views of other tensors, whose last stride says nothing."""
    import torch
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    b = A.Batch(i(4, 3)[::4, ::3], i(8)[::8], i(2), tokens=5, max_new=5, max_len=9)
    assert b.desc.table_stride == 1 and b.sequences == 1
    assert A.Score(0.1, prefix=i(7)[::7], doc=i(3, 9)[:1, ::9]).sequences == 1
    with pytest.raises(TypeError):
        A.Batch(i(4, 6)[:, ::3], i(4), max_len=9)
