"""A step's tables built on the GPU against plain loops: every output is an integer and has to be equal."""
import numpy as np
import pytest

from oracle import bwla_cache8_oracle as orc

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    pytest.importorskip("torch")                       # (in front of the library: one HIP runtime for both)
    from paper_2605_00422_amd import attention_binding
    attention_binding.load()
    return attention_binding


class Step:
    """Requests whose pages lie anywhere, and a ring of the free ones whose front is anywhere."""

    def __init__(self, lens, new, page=16, done=None, shift=None, tokens=None, spare=3, columns=None, capacity=None, seed=0, gone=()):
        rng = np.random.default_rng(seed)
        n = len(lens)
        self.page, self.lens, self.new, self.done, self.shift = page, np.array(lens), np.array(new), done, shift
        held = [-(-max(int(x), 0) // page) for x in lens]
        after = [-(-((0 if done is not None and done[b] else max(int(lens[b]), 0)) + max(int(new[b]), 0)) // page) for b in range(n)]
        self.columns = columns or max(held + after + [1])
        need = sum(max(a - (0 if done is not None and done[b] else h), 0) for b, (a, h) in enumerate(zip(after, held)))
        self.count = max(need + spare, 0)
        self.pages = sum(held) + self.count
        capacity = self.pages + 5 if capacity is None else capacity
        order = rng.permutation(self.pages).astype(np.int32)
        self.table = np.full((n, self.columns), -7, np.int32)
        at = 0
        for b in range(n):
            self.table[b, :held[b]] = order[at:at + held[b]]
            at += held[b]
        for b, e in gone:
            self.table[b, e] = -1
        self.front = int(rng.integers(0, capacity))
        self.ring = np.full(capacity, -9, np.int32)
        self.ring[(self.front + np.arange(self.count)) % capacity] = order[at:]
        self.tokens = int(np.maximum(self.new, 0).sum()) + 4 if tokens is None else tokens
        self.max_len = self.columns * page

    def run(self, A, in_place=False, outputs=True, ws=None):
        import torch
        i32 = lambda x: None if x is None else torch.tensor(np.asarray(x), dtype=torch.int32).cuda()  # noqa: E731
        n = len(self.lens)
        table, ring, state, length = i32(self.table), i32(self.ring), i32([self.front, self.count]), i32(self.lens)
        full = lambda m, t=torch.int32: torch.full((m,), 77, dtype=t, device="cuda")  # noqa: E731
        out = {"table": table, "ring": ring, "state": state if in_place else full(2), "length": length if in_place else full(n),
               "first": full(n + 1), "status": full(4)}
        more = {"position": full(self.tokens), "slot": full(self.tokens, torch.int64), "sequence": full(self.tokens)} if outputs else {}
        pool = A.PagePool(ring, state, self.page, None if in_place else out["state"], pages=self.pages)
        need = max(16, A.batch_build_workspace_size(n, self.tokens))
        ws = torch.full((need,), 0xff, dtype=torch.uint8, device="cuda") if ws is None else ws
        A.batch_build(pool, table, length, i32(self.new), out["length"], out["first"], out["status"], self.tokens, self.max_len, i32(self.done),
                      i32(self.shift), ws=ws, **more)
        return {k: v.cpu().numpy() for k, v in {**out, **more}.items()}

    def want(self):
        return orc.build(self.lens, self.new, self.table, self.ring, [self.front, self.count], self.page, self.pages, self.tokens, self.max_len,
                         self.done, self.shift)

    def check(self, A, **kw):
        got, want = self.run(A, **kw), self.want()
        for k, v in got.items():
            assert np.array_equal(v, want[k]), (k, v, want[k])
        return got


def random_step(n, seed, most=300, done=True, **kw):
    rng = np.random.default_rng(seed)
    return Step(rng.integers(0, most, n), rng.choice([0, 1, 1, 1, 2, 40], n), done=rng.integers(0, 4, n) == 0 if done else None,
                shift=rng.integers(-3, 50, n), seed=seed, **kw)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("n,page", [(1, 8), (2, 16), (63, 16), (64, 64), (65, 8), (1000, 16), (1024, 16), (1025, 16), (3000, 8), (2048, 128), (5000, 16)])
def test_requests_of_all_ages(A, n, page, in_place):
    random_step(n, seed=n, page=page).check(A, in_place=in_place)


@pytest.mark.parametrize("n", [7, 2000])
def test_without_options(A, n):
    random_step(n, seed=3, done=False).check(A, outputs=False)
    s = random_step(n, seed=4, done=False)
    s.shift = None
    s.check(A)


@pytest.mark.parametrize("lens,new,done", [
    ([0], [1], None), ([0], [0], None), ([16], [1], None), ([15], [1], None), ([17], [0], [1]), ([16, 32], [16, 0], [1, 1]),
    ([1, 0, 5], [0, 0, 0], None), ([40, 40], [5, 5], [0, 1]), ([33], [8192], [1]), ([5], [9000], None)])
def test_edges(A, lens, new, done):
    Step(lens, new, done=done).check(A)


def test_nothing_at_all(A):
    s = Step([], [], tokens=3)
    s.table = np.zeros((0, 1), np.int32)
    s.check(A)
    Step([3], [0], tokens=0).check(A)


@pytest.mark.parametrize("n", [20, 1500])
def test_prompts_of_many_rows(A, n):
    rng = np.random.default_rng(1)
    new = rng.choice([0, 1, 1, 700], n)
    new[3] = 20000
    Step(rng.integers(0, 100, n), new, done=rng.integers(0, 3, n) == 0, seed=8).check(A)


@pytest.mark.parametrize("n", [50, 1200])
@pytest.mark.parametrize("kw", [dict(spare=-1), dict(spare=-1000000), dict(tokens=5)])
def test_what_does_not_fit_changes_nothing_but_what_is_done(A, n, kw):
    s = random_step(n, seed=17, **kw)
    got = s.check(A)
    assert got["status"][:3].any() and not got["first"].any() and (got["position"] == -1).all()
    same = np.ones(n, bool) if s.done is None else ~np.asarray(s.done, bool)
    assert np.array_equal(got["length"][same], s.lens[same])
    assert np.array_equal(got["table"], s.table)


@pytest.mark.parametrize("n", [4, 1100])
def test_requests_longer_than_max_len(A, n):
    s = random_step(n, seed=5)
    s.new[n // 2] = s.max_len + 1
    s.tokens += s.max_len + 1
    got = s.check(A)
    assert got["status"][1] >= 1 and not got["first"].any()


@pytest.mark.parametrize("n", [6, 1300])
def test_lengths_and_new_tokens_outside_their_bounds(A, n):
    s = random_step(n, seed=6)
    s.lens[0], s.new[1], s.new[2] = -5, -3, 0
    s.lens[3] = 1 << 30                                 # cut to max_len
    s.done = np.zeros(n, bool)
    s.done[3] = True
    s.new[4] = 2 ** 31 - 1 if n > 1000 else s.new[4]    # (sums beyond 32 bits)
    s.new[5] = 2 ** 31 - 1 if n > 1000 else s.new[5]
    s.check(A)


@pytest.mark.parametrize("n", [5, 1300])
def test_pages_given_back_leave_out_what_names_none(A, n):
    lens = np.full(n, 100)
    gone = [(b, e) for b in range(n) for e in range(7) if (b + e) % 3 == 0]
    s = Step(lens, np.ones(n, int), done=np.arange(n) % 2, gone=gone, seed=2)
    s.table[1, 1] = s.pages + 3
    s.check(A)


def test_a_ring_that_is_full_keeps_what_it_holds(A):
    s = Step([64] * 8, [0] * 8, done=[1] * 8, spare=2, capacity=20)
    got = s.check(A)
    assert got["state"][1] == 20


@pytest.mark.parametrize("state", [(-3, 5), (1 << 30, 1 << 30), (0, -1)])
def test_a_state_that_is_none(A, state):
    s = Step([5, 20], [1, 1], spare=30)
    s.front, s.count = state
    s.ring[:] = np.arange(len(s.ring)) % s.pages
    s.check(A)


def test_the_steps_of_a_server(A):
    """Requests come, grow and go for many steps, in place: no page is ever named twice."""
    import torch
    rng = np.random.default_rng(0)
    n, page, pages, columns = 37, 16, 400, 20
    pool = A.PagePool.full(pages, page)
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32).cuda()  # noqa: E731
    table, length = torch.full((n, columns), -1, dtype=torch.int32, device="cuda"), i32([0] * n)
    first, status, ws = i32([0] * (n + 1)), i32([0] * 4), torch.empty(4096, dtype=torch.uint8, device="cuda")
    refused = 0
    for step in range(60):
        new, done = rng.choice([0, 1, 1, 1, 30, 90], n), rng.random(n) < 0.15
        before = length.cpu().numpy()
        new = np.minimum(new, columns * page - np.where(done, 0, before))
        A.batch_build(pool, table, length, i32(new), length, first, status, 4000, columns * page, i32(done), ws=ws)
        missing, lens = status.cpu().numpy(), length.cpu().numpy()
        assert missing[1] == missing[2] == 0
        refused += missing[0] > 0
        assert np.array_equal(lens, np.where(done, 0, before) + (new if missing[0] == 0 else 0))
        front, count = pool.state.cpu().numpy()
        t, ring = table.cpu().numpy(), pool.ring.cpu().numpy()
        used = [p for b in range(n) for p in t[b, :-(-lens[b] // page)]]
        free = [ring[(front + i) % pages] for i in range(count)]
        assert sorted(used + free) == list(range(pages))
    assert 0 < refused < 60


def test_captured_and_replayed(A):
    """A captured step advances the requests at each replay as eager calls do."""
    import torch
    n, page, pages = 9, 16, 200
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32).cuda()  # noqa: E731

    def fresh():
        return dict(pool=A.PagePool.full(pages, page), table=torch.full((n, 12), -1, dtype=torch.int32, device="cuda"), length=i32([0] * n),
                    new=i32([17] + [1] * (n - 1)), first=i32([0] * (n + 1)), status=i32([0] * 4), slot=torch.zeros(30, dtype=torch.int64, device="cuda"))

    def call(s):
        A.batch_build(s["pool"], s["table"], s["length"], s["new"], s["length"], s["first"], s["status"], 30, 192, slot=s["slot"], ws=ws)

    ws = torch.empty(4096, dtype=torch.uint8, device="cuda")
    one, two = fresh(), fresh()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call(two)
    torch.cuda.synchronize()
    two = fresh()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(two)
    torch.cuda.synchronize()
    for _ in range(12):                                # (the last ones do not fit: requests longer than 192)
        call(one)
        graph.replay()
        torch.cuda.synchronize()
        for k in ("table", "length", "first", "status", "slot"):
            assert torch.equal(one[k], two[k]), k
        assert torch.equal(one["pool"].state, two["pool"].state) and torch.equal(one["pool"].ring, two["pool"].ring)
    assert one["status"][1] > 0


@pytest.mark.parametrize("tokens", [3, 5000])
def test_no_requests_but_rows(A, tokens):
    s = Step([], [], tokens=tokens)
    s.table = np.zeros((0, 1), np.int32)
    s.check(A)


@pytest.mark.parametrize("n", [256, 257, 320, 65535])
def test_many_requests(A, n):
    rng = np.random.default_rng(n)
    Step(rng.integers(0, 40, n), rng.integers(0, 3, n), done=rng.integers(0, 9, n) == 0, seed=n).check(A)
