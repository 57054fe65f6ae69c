"""A serving step as it is used: tables built on the GPU, normed and turned rows into a cache in 8 bits, attention over it; and the block
that runs it between two layers."""
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


def steps(rng, places, count, longest):
    """(new tokens, done) of each step: requests of random prompts and lengths."""
    left = [0] * places
    for _ in range(count):
        done = [int(n == 0) for n in left]
        new = [int(rng.integers(1, longest)) if d else 1 for d in done]
        left = [int(rng.integers(2, 9)) if d else n - 1 for d, n in zip(done, left)]
        yield new, done


@pytest.mark.parametrize("code", ["i8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_steps_of_a_server_against_the_oracle(A, code, dtype):
    """Each step's attention against the oracle over the values that the cache stands for, and those values against every token that was
    ever written, to a step of the page's scale."""
    import torch
    from paper_2605_00422_amd.attention_block import Requests, tables
    T = torch.bfloat16 if dtype == "bf16" else torch.float32
    hq, hkv, d, page, places, max_len = 4, 2, 64, 16, 3, 112
    cache = A.KVCache8.empty(21, hkv, page, d, T, torch.int8 if code == "i8" else torch.float8_e4m3fn)
    plain = A.KVCache(*(torch.zeros(21, hkv, page, d, device="cuda") for _ in range(2)))      # the same rows as they are, in fp32
    rope, requests = tables(torch, max_len, d, "cuda"), Requests(places, max_len, 21, page)
    norm = A.HeadNorm(torch.rand(d, generator=torch.Generator().manual_seed(1)).cuda() + 0.5, None)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    rng, gen = np.random.default_rng(5), torch.Generator(device="cuda").manual_seed(2)
    for new, done in steps(rng, places, 14, 100):
        batch, position = requests.step(i32(new), i32(done), rows=sum(new) + 2, most=max(new))
        qkv = torch.randn(sum(new) + 2, (hq + 2 * hkv) * d, generator=gen, device="cuda")
        q, out = (torch.zeros(sum(new) + 2, hq, d, dtype=T, device="cuda") for _ in range(2))
        A.norm_rope_append(cache, batch, rope, norm, qkv, position, q)
        wide = torch.zeros(sum(new) + 2, hq, d, device="cuda")
        A.norm_rope_append(plain, batch, rope, norm, qkv, position, wide)
        ws = torch.empty(max(16, A.attention8_workspace_size(cache, batch, hq)), dtype=torch.uint8, device="cuda")
        A.attention8_forward(cache, batch, A.Score(d ** -0.5), q, out, None, ws)
        k, v = (torch.empty(places, max_len, hkv, d, device="cuda") for _ in range(2))
        A.cache8_read(cache, batch, k, v)
        assert requests.status.tolist() == [0, 0, 0, sum(new)]
        assert not out[sum(new):].any()                                          # (rows of no request are left as they were)
        first, lens, table = requests.first.tolist(), requests.length.tolist(), requests.table.cpu().numpy()
        for b in range(places):
            n, m = lens[b], new[b]
            kb, vb = (t[b, :n].double().cpu().numpy() for t in (k, v))
            rows = slice(first[b], first[b] + m)
            want, _, _, vabs, qk, top = orc.attend(q[rows].double().cpu().numpy(), kb, vb, d ** -0.5)
            eps = 2 * (d + 4) * U * qk + 8 * U * top + 2.0 ** -38 * d * 8 * np.abs(kb).max()
            rel = np.expm1(2 * eps) + (2 * n + 24) * U
            # (values come back as fp32 products: u of each besides)
            bound = vabs * (rel[..., None] + 2 * U + (2.0 ** -11 if dtype == "bf16" else 2.0 ** -22)) + n * 2.0 ** -35 * np.abs(vb).max()
            bound = bound + np.abs(want) * (2.0 ** -8 if dtype == "bf16" else 4 * U)
            assert np.all(np.abs(out[rows].double().cpu().numpy() - want) <= bound)
            pages = table[b][np.arange(n) // page]
            for t, scale, mine in ((plain.k, cache.k_scale, kb), (plain.v, cache.v_scale, vb)):
                was = t[pages, :, np.arange(n) % page].double().cpu().numpy()
                s = scale[pages].double().cpu().numpy()[..., None]
                step = s if code == "i8" else s * 2.0 ** np.maximum(np.floor(np.log2(np.maximum(np.abs(was / s), 1e-30))) - 3, -9)
                assert np.all(np.abs(was - mine) <= step * 1.0001 + 4 * U * np.abs(was))


@pytest.mark.parametrize("code", ["i8", "e4m3"])
def test_a_decoding_step_captured_with_its_tables(A, code):
    """Tables, append and attention in one graph: every replay is a step, as eager calls on a copy of the state make it."""
    import torch
    from paper_2605_00422_amd.attention_block import Requests, tables
    hq, hkv, d, page, places = 8, 2, 128, 16, 5
    rope, norm = tables(torch, 200, d, "cuda"), A.HeadNorm()
    gen = torch.Generator(device="cuda").manual_seed(3)

    class Side:
        def __init__(self):
            self.cache = A.KVCache8.empty(60, hkv, page, d, torch.bfloat16, torch.int8 if code == "i8" else torch.float8_e4m3fn)
            self.requests = Requests(places, 160, 60, page)
            self.new = torch.ones(places, dtype=torch.int32, device="cuda")
            self.q, self.out = (torch.zeros(places, hq, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            self.ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")

        def step(self, qkv):
            batch, position = self.requests.step(self.new)
            A.norm_rope_append(self.cache, batch, rope, norm, qkv, position, self.q)
            A.attention8_forward(self.cache, batch, A.Score(d ** -0.5), self.q, self.out, None, self.ws)

    eager, held = Side(), Side()
    qkv = torch.randn(places, (hq + 2 * hkv) * d, generator=gen, device="cuda")
    warm = Side()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        warm.step(qkv)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held.step(qkv)
    for i in range(40):
        qkv.copy_(torch.randn(qkv.shape, generator=gen, device="cuda") * (1 + i % 7))
        graph.replay()
        eager.step(qkv)
        torch.cuda.synchronize()
        assert torch.equal(held.out, eager.out) and torch.equal(held.q, eager.q)
        assert torch.equal(held.cache.k.view(torch.uint8), eager.cache.k.view(torch.uint8)) and torch.equal(held.cache.v_scale, eager.cache.v_scale)
        assert held.requests.length.tolist() == [i + 1] * places


def test_the_block_runs_the_calls_one_by_one(A):
    """A block with a cache in 8 bits and normed heads gives what its calls give, to the bit; with one as it is and normed heads too."""
    import torch
    from paper_2605_00422_amd import binding as B
    from paper_2605_00422_amd.attention_block import AttentionBlock, random_layer, tables
    gen = torch.Generator(device="cuda").manual_seed(7)
    hidden, hq, hkv, d = 256, 4, 2, 64
    qkv_layer, o_layer = random_layer(torch, gen, (hq + 2 * hkv) * d, hidden, 8, "cuda"), random_layer(torch, gen, hidden, hq * d, 8, "cuda")
    rope, norm = tables(torch, 64, d, "cuda"), A.HeadNorm(torch.rand(hq, d, generator=gen, device="cuda") + 0.5, torch.rand(hkv, d, generator=gen, device="cuda") + 0.5)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    for eight in (True, False):
        def cache():
            if eight:
                return A.KVCache8.empty(6, hkv, 16, d, torch.bfloat16)
            return A.KVCache(*(torch.zeros(6, hkv, 16, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)))
        one, two = cache(), cache()
        block = AttentionBlock(qkv_layer, o_layer, one, rope, hq, norm=norm)
        table, length = i32([[4, 1, 0], [2, 3, 5]]), i32([40, 7])
        for news, lens in (([40, 7], [40, 7]), ([1, 1], [41, 8])):
            n = sum(news)
            batch = A.Batch(table, i32(lens), i32([0, news[0], n]), tokens=n, max_new=max(news), max_len=48)
            x = torch.randn(n, hidden, generator=gen, device="cuda").bfloat16()
            position = i32([[i for m, t in zip(lens, news) for i in range(m - t, m)]])
            y = block(x, batch, position, torch.empty(n, hidden, device="cuda"))
            qkv, q, out = torch.empty(n, (hq + 2 * hkv) * d, device="cuda"), *(torch.empty(n, hq, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            B.decode_forward(qkv_layer, x, B.Activations(qkv_layer, n), qkv)
            A.norm_rope_append(two, batch, rope, norm, qkv, position, q)
            ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
            (A.attention8_forward if eight else A.attention_forward)(two, batch, A.Score(d ** -0.5), q, out, ws=ws)
            want = B.decode_forward(o_layer, out.view(n, -1), B.Activations(o_layer, n), torch.empty(n, hidden, device="cuda"))
            assert torch.equal(y, want) and torch.isfinite(y).all()
        if eight:
            for wrong in (lambda: block(x, batch, position, y, watch=True), lambda: block.cut(batch, table, 8, 1, 1, length),
                          lambda: block.watch_last(batch, batch)):
                with pytest.raises(ValueError, match="sums"):
                    wrong()


@pytest.mark.parametrize("code", ["i8", "e4m3"])
def test_the_command_runs(A, code):
    import torch
    from paper_2605_00422_amd.attention_block import serve
    outputs, lengths = serve(code)
    assert len(outputs) == 24 and all(torch.isfinite(y).all() for y in outputs) and lengths.min() > 0 and lengths.max() <= 160


def test_other_streams(A):
    """The call runs on the current stream, behind what that stream has."""
    import torch
    cache = A.KVCache8.empty(8, 2, 16, 64, torch.bfloat16)
    cache.k_scale.fill_(0.01), cache.v_scale.fill_(0.01)
    cache.v.fill_(1)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    batch = A.Batch(i32([[1, 2, 3]]), i32([40]), max_len=40)
    q, out, slow = torch.zeros(1, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(1 << 26, device="cuda")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(20):
            slow.add_(1)
        cache.v.fill_(100)
        A.attention8_forward(cache, batch, A.Score(0.1), q, out)
    side.synchronize()
    assert (out.float() - 1.0).abs().max() <= 2.0 ** -8


def test_steps_of_many_sizes_share_one_room(A):
    """Positions of steps of fewer rows lie where those of the longest lie; what a longer step outgrew stays as a captured one knows it."""
    import torch
    from paper_2605_00422_amd.attention_block import Requests
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    r, length = Requests(3, 400, 90, 16), [0, 0, 0]
    seen = {}
    for new in ([1, 1, 1], [2, 0, 9], [60, 1, 30], [1, 1, 1], [5, 70, 0]):
        _, position = r.step(i32(new), rows=sum(new), most=max(new))
        assert position.shape == (1, sum(new))
        want = [n + i for n, m in zip(length, new) for i in range(m)]
        assert position[0].tolist() == want
        length = [n + m for n, m in zip(length, new)]
        seen.setdefault(position.data_ptr(), []).append(sum(new))
    assert list(seen.values()) == [[3], [11], [91, 3, 75]] and len(r._room) == 3
