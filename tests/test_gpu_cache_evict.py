"""Eviction from long caches: a kernel for each range of lengths, at the ranges' ends and inside, against the fp64 oracle.  Equal in
every bit: the kept tokens, their number, positions, keys, values and sums, and whatever is not written."""
import numpy as np
import pytest

from oracle import bwla_attention_oracle as orc

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    pytest.importorskip("torch")                       # (in front of the library: one HIP runtime for both)
    from paper_2605_00422_amd import attention_binding
    attention_binding.load()
    return attention_binding


@pytest.mark.parametrize("max_len", [2047, 2048, 2049, 3001, 4096, 4097, 8191, 8193, 16384, 16385, 32768, 32769, 40963])
@pytest.mark.parametrize("dtype,part,sinks,recent", [("bf16", 0.3, 4, 100), ("f32", 0.95, 0, 0), ("bf16", 2.0, 3, 3), ("f32", 0.0, 0, 1), ("bf16", 0.6, 700, 900)])
def test_eviction_from_long_caches(A, dtype, max_len, part, sinks, recent):
    import torch
    rng = np.random.default_rng(max_len)
    page, hkv, d, n = 16, 2, 8, 5
    lens = np.array([max_len, max_len // 3, max_len - 1023, 5, 0])
    keep = int(max_len * part) + 1
    recent = min(recent, keep - sinks)
    per, per_out = -(-max_len // page), -(-min(keep, max_len) // page)
    pages = n * (per + per_out) + 2
    order = rng.permutation(pages).astype(np.int32)
    table, table_out = order[:n * per].reshape(n, per), order[n * per:n * (per + per_out)].reshape(n, per_out)
    stored = table.copy()
    gone = rng.random(table.shape) < 0.05              # pages that do not exist
    table[gone] = np.where(rng.random(table.shape) < 0.5, -1, pages + 3)[gone]
    # few different sums, many equal ones, and some that are no numbers, or infinite
    w = np.floor(rng.exponential(1.0, (pages, hkv, page)) * 3).astype(np.float32) / 4
    odd = rng.random(w.shape)
    w[odd < 0.003], w[(odd > 0.1) & (odd < 0.102)], w[(odd > 0.2) & (odd < 0.202)] = np.nan, np.inf, -np.inf
    w[(odd > 0.3) & (odd < 0.35)] *= -1
    T = torch.bfloat16 if dtype == "bf16" else torch.float32
    k, v = (torch.from_numpy(rng.standard_normal((pages, hkv, page, d)).astype(np.float32)).to(T).cuda() for _ in range(2))
    k0, v0 = (x.float().cpu().numpy() for x in (k, v))
    i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda()  # noqa: E731
    pos = rng.integers(0, 1 << 30, (n, max_len + 1))
    sums, length = torch.from_numpy(w).cuda(), torch.full((n,), -9, dtype=torch.int32, device="cuda")
    kept, pos_out = (torch.full((n, keep), -9, dtype=torch.int32, device="cuda") for _ in range(2))
    cache, batch = A.KVCache(k, v), A.Batch(i32(table), i32(lens), max_len=max_len)
    ws = torch.full((A.cache_evict_workspace_size(cache, batch),), 0xff, dtype=torch.uint8, device="cuda")
    A.cache_evict(cache, batch, i32(table_out), sums, keep, sinks, recent, length, kept, i32(pos), pos_out, ws)
    k1, v1, w1 = k0.copy(), v0.copy(), w.copy()
    for b, m in enumerate(lens):
        j = np.arange(m)
        there = ~gone[b, j // page]
        with np.errstate(invalid="ignore"):
            want = orc.kept(np.where(there[:, None], w[stored[b, j // page], :, j % page], 0), keep, sinks, recent, there)
        assert int(length[b]) == len(want)
        assert np.array_equal(kept[b].cpu().numpy(), np.pad(want, (0, keep - len(want)), constant_values=-1))
        assert np.array_equal(pos_out[b].cpu().numpy(), np.pad(pos[b, want], (0, keep - len(want)), constant_values=-1))
        i, frm, to = np.arange(len(want)), stored[b, want // page], table_out[b, np.arange(len(want)) // page]
        for new, old in ((k1, k0), (v1, v0), (w1, w)):
            new[to, :, i % page] = old[frm, :, want % page]
    for got, new in ((k, k1), (v, v1), (sums, w1)):
        assert np.array_equal(got.float().cpu().numpy(), new, equal_nan=True)
