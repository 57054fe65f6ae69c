"""What an attention block holds on to: its memory, the addresses of captured calls, the queries of the call before."""
import pytest

pytestmark = pytest.mark.gpu
HQ, HKV, D, PAGE, HIDDEN = 4, 2, 64, 16, 512


@pytest.fixture(scope="module")
def A():
    pytest.importorskip("torch")                       # (in front of the library: one HIP runtime for both)
    from paper_2605_00422_amd import attention_binding
    attention_binding.load()
    return attention_binding


def i32(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.fixture
def make(A):
    def make(pages=160, **kw):
        import torch
        from paper_2605_00422_amd import attention_block as T
        gen = torch.Generator(device="cuda").manual_seed(5)
        k, v = (torch.zeros(pages, HKV, PAGE, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        block = T.AttentionBlock(T.random_layer(torch, gen, (HQ + 2 * HKV) * D, HIDDEN, 8, "cuda"),
                                 T.random_layer(torch, gen, HIDDEN, HQ * D, 8, "cuda"), A.KVCache(k, v), T.tables(torch, 2000, D, "cuda"), HQ, **kw)

        def prompt(m, page0=0, watch=True):
            """m rows from page page0 on: (input, batch, position, output)."""
            batch = A.Batch(i32([list(range(page0, page0 + -(-m // PAGE)))]), i32([m]), i32([0, m]), tokens=m, max_new=m, max_len=m)
            x, y = torch.randn(m, HIDDEN, generator=gen, device="cuda").bfloat16(), torch.empty(m, HIDDEN, device="cuda")
            block(x, batch, i32([list(range(m))]), y, watch=watch)
            return x, batch, y
        return block, prompt, gen
    return make


def test_calls_of_all_lengths_do_not_add_up(make):
    import torch
    block, prompt, _ = make()
    prompt(300)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    for m in range(1, 300, 7):
        prompt(m)
    assert torch.cuda.memory_allocated() <= before + (1 << 16)
    prompt(301)                                        # twice as much once, and then no more for a while
    before = torch.cuda.memory_allocated()
    for m in range(302, 600, 7):
        prompt(m)
    assert block.rows == 600 and torch.cuda.memory_allocated() <= before + (1 << 16)


@pytest.mark.parametrize("own", [False, True])
def test_a_captured_step_outlives_larger_calls(A, make, own):
    """A decoding step behind 700 tokens, whose cache is divided over workgroups: replays give what the same step gives outside the graph,
    whatever the block did in between."""
    import torch
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda") if own else None
    block, prompt, gen = make(ws=ws)
    prompt(700)
    step = A.Batch(i32([list(range(44))]), i32([701]), max_len=704)
    assert A.attention_workspace_size(block.cache, step, HQ, True) > 0
    x, y, position = torch.randn(1, HIDDEN, generator=gen, device="cuda").bfloat16(), torch.empty(1, HIDDEN, device="cuda"), i32([[700]])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block(x, step, position, y)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block(x, step, position, y)
    length, table_out = i32([0, 0]), i32([[150, 151], [152, 153]])
    for i in range(4):
        _, batch, _ = prompt(900 + 40 * i, page0=50, watch=False)
        block.watch_last(batch, A.Batch(batch.table, batch.length, i32([0, 20]), tokens=20, max_new=20, max_len=batch.max_len))
        both = A.Batch(i32([list(range(44)), list(range(50, 94))]), i32([700, 700]), max_len=704)
        block.cut(both, table_out, 32, 2, 8, length)
        held = [torch.full((1 << 20,), 7.0, device="cuda") for _ in range(4)]  # (what a replay must not write to)
        x.mul_(-1)
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        block(x, step, position, y)
        assert torch.equal(got, y) and all((h == 7).all() for h in held)


def test_what_a_block_refuses(A, make):
    import torch
    from paper_2605_00422_amd import binding as B
    block, prompt, gen = make()
    _, first, _ = prompt(64, watch=False)
    last = lambda b, n: A.Batch(b.table, b.length, i32([0, n]), tokens=n, max_new=n, max_len=b.max_len)  # noqa: E731
    with pytest.raises(ValueError):
        block.watch_last(first, last(first, 65))
    _, second, _ = prompt(64, page0=8, watch=False)    # as many rows: the first one's queries are gone
    with pytest.raises(ValueError):
        block.watch_last(first, last(first, 8))
    block.watch_last(second, last(second, 8))
    block, prompt, gen = make(ws=torch.empty(16, dtype=torch.uint8, device="cuda"))
    prompt(200, watch=False)                           # (one part of the cache, no sums: no scratch)
    step = A.Batch(i32([list(range(44))]), i32([701]), max_len=704)
    with pytest.raises(B.BwlaError):
        block(torch.zeros(1, HIDDEN, dtype=torch.bfloat16, device="cuda"), step, i32([[700]]), torch.empty(1, HIDDEN, device="cuda"))
