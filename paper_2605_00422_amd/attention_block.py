"""The attention half of a decoder block on W1A6 layers: x -> q|k|v projection -> rotary positions into the paged cache ->
attention -> o projection, for prompts and for decoding steps, with the cache cut to a budget by the weights that its tokens got.

    python -m paper_2605_00422_amd.attention_block

runs a small block of random weights: two prompts, a cut of their caches, sixteen decoding steps.  Every step is a kernel of the
library; torch holds the memory.  Tables, lengths and pages are the caller's (a serving loop's scheduler), and so is what a
residual or a norm adds around it."""
from __future__ import annotations

from . import attention_binding as A, binding as B


class AttentionBlock:
    """qkv, o: PackedLayer of the merged projection ((q_heads + 2 kv_heads) head_dim rows) and of the output.  cache: KVCache,
    bfloat16.  Scores: scale (default head_dim^-1/2), and what else Score takes, per call.
    rows: of a call, that room is made for at the start; a call of more makes room for twice as many as before at least, and what was
    there stays, where captured calls find it (so that all of it is a few times the longest call's).  ws: uint8, scratch of all calls, which
    raise BwlaError where it is too small for them (attention_binding.*_workspace_size say what they want); without it each takes its own
    from torch's allocator, a captured call from the graph's.  A block serves one stream at a time."""

    def __init__(self, qkv, o, cache: A.KVCache, rope: A.Rope, q_heads: int, scale=None, rows: int = 64, ws=None):
        d = cache.head_dim
        if qkv.desc.N != (q_heads + 2 * cache.kv_heads) * d or o.desc.K != q_heads * d:
            raise ValueError("qkv must have (q_heads + 2 kv_heads) head_dim rows, o q_heads head_dim columns")
        self.qkv, self.o, self.cache, self.rope, self.q_heads = qkv, o, cache, rope, q_heads
        self.scale = d ** -0.5 if scale is None else scale
        self.sums = cache.weights()                    # of the softmax weights that each cached token got
        self._room, self._rows, self._last, self._ws = [], {}, None, ws
        self._make(rows)

    def _make(self, M):
        import torch
        c = self.cache
        new = lambda *s, t=torch.float32: torch.empty(M, *s, dtype=t, device=c.k.device)  # noqa: E731
        self.rows = M
        self._room.append((B.Activations(self.qkv, M), new(self.qkv.desc.N), new(self.q_heads, c.head_dim, t=c.dtype),
                           new(self.q_heads, c.head_dim, t=c.dtype), new(self.q_heads), B.Activations(self.o, M)))

    def _scratch(self, size, *args):
        """size(*args) bytes, where the caller gave none."""
        if self._ws is not None:
            return self._ws
        import torch
        return torch.empty(max(size(*args), 16), dtype=torch.uint8, device=self.cache.k.device)

    def _buffers(self, M):
        """What a call of M rows writes on the way: the first rows of the room (kept as views until a call of another number)."""
        if M not in self._rows:
            if M > self.rows:
                self._make(max(M, 2 * self.rows))
            act_in, qkv, q, out, lse, act_out = self._room[-1]
            self._rows = {M: (act_in, qkv[:M], q[:M], out[:M], lse[:M], act_out)}
        return self._rows[M]

    def __call__(self, x, batch: A.Batch, position, y, watch: bool = True, **score):
        """x (tokens, columns of qkv), bfloat16 or float32 -> y (tokens, rows of o), float32.  position: int32 (axes, tokens).
        watch: whether the weights that this call's queries give count; the new tokens' sums start at zero either way."""
        act_in, qkv, q, out, lse, act_out = self._buffers(x.shape[0])
        self._last = batch
        score = A.Score(self.scale, **score)
        B.decode_forward(self.qkv, x, act_in, qkv)
        A.rope_append(self.cache, batch, self.rope, qkv, position, q, self.sums)
        ws = self._scratch(A.attention_workspace_size, self.cache, batch, self.q_heads, watch)
        A.attention_forward(self.cache, batch, score, q, out, lse, self.sums if watch else None, ws)
        return B.decode_forward(self.o, out.view(x.shape[0], -1), act_out, y)

    def watch_last(self, batch: A.Batch, last: A.Batch, **score):
        """The sums of weights of a long prompt's last queries alone: batch was the call before, of one sequence (watch=False), whose queries
        are still there; last is the same sequence with its last tokens as the new ones."""
        if batch is not self._last:
            raise ValueError("batch is not that of the call before: its queries are gone")
        if batch.sequences != 1 or last.sequences != 1 or last.tokens > batch.tokens:
            raise ValueError("one sequence, and the last of its rows")
        _, _, q, _, lse, _ = self._rows[batch.tokens]
        ws = self._scratch(A.attention_weights_workspace_size, self.cache, last, self.q_heads)
        A.attention_weights(self.cache, last, A.Score(self.scale, **score), q[batch.tokens - last.tokens:],
                            lse[batch.tokens - last.tokens:], self.sums, ws)

    def cut(self, batch: A.Batch, table_out, keep: int, sinks: int, recent: int, length_out):
        """Each sequence's `keep` tokens with the largest sums, its first and last ones among them, to the pages of table_out."""
        ws = self._scratch(A.cache_evict_workspace_size, self.cache, batch)
        return A.cache_evict(self.cache, batch, table_out, self.sums, keep, sinks, recent, length_out, ws=ws)


def random_layer(torch, gen, N, K, rank, dev):
    """A packed layer of random weights, its columns rotated by random orthogonal factors."""
    n1, n2 = B.kron_factor(K)
    f32 = lambda *s: torch.randn(*s, generator=gen, device=dev)  # noqa: E731
    R1, R2 = (torch.linalg.qr(torch.randn(n, n, generator=torch.Generator().manual_seed(n)))[0].contiguous().to(dev) for n in (n1, n2))
    return B.pack_weights(f32(N, K) * K ** -0.5, R1, R2, f32(K, rank) * 0.02, f32(N, rank) * 0.02, n1, n2)


def tables(torch, rows, dim, dev, base=10000.0):
    at = torch.arange(rows, dtype=torch.float64)[:, None] * base ** (-torch.arange(dim // 2, dtype=torch.float64) / (dim // 2))
    return A.Rope(at.cos().float().to(dev), at.sin().float().to(dev))


def main(hidden=512, q_heads=8, kv_heads=2, dim=64, page=16, prompts=(300, 77), keep=64, steps=16, dev="cuda"):
    """Returns the outputs of the prompts and of the steps, and the cached lengths of the steps."""
    import torch
    gen = torch.Generator(device=dev).manual_seed(1)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
    per, n = -(-max(prompts) // page), len(prompts)
    after = -(-(keep + steps) // page)                 # pages of a sequence behind the cut
    k, v = (torch.zeros(n * (per + after), kv_heads, page, dim, dtype=torch.bfloat16, device=dev) for _ in range(2))
    block = AttentionBlock(random_layer(torch, gen, (q_heads + 2 * kv_heads) * dim, hidden, 8, dev),
                           random_layer(torch, gen, hidden, q_heads * dim, 8, dev),
                           A.KVCache(k, v), tables(torch, max(prompts) + steps, dim, dev), q_heads)
    outputs, lengths = [], []
    table, length = i32([[b * per + p for p in range(per)] for b in range(n)]), i32(list(prompts))
    for b, m in enumerate(prompts):                    # the prompts; the weights of all queries count, of a long one the last 32
        batch = A.Batch(table[b:b + 1], length[b:b + 1], i32([0, m]), tokens=m, max_new=m, max_len=m)
        x, y = torch.randn(m, hidden, generator=gen, device=dev).bfloat16(), torch.empty(m, hidden, device=dev)
        block(x, batch, i32([list(range(m))]), y, watch=m <= 128)
        if m > 128:
            block.watch_last(batch, A.Batch(table[b:b + 1], length[b:b + 1], i32([0, 32]), tokens=32, max_new=32, max_len=m))
        outputs.append(y)
    # their caches cut to the heaviest tokens, in fresh pages
    table_out, kept = i32([[n * per + b * after + p for p in range(after)] for b in range(n)]), i32([0] * n)
    block.cut(A.Batch(table, length, max_len=max(prompts)), table_out, keep, 4, 16, kept)
    # decoding: a token of each sequence a step, at the position behind its last one
    step, y = A.Batch(table_out, kept, max_len=keep + steps), torch.empty(n, hidden, device=dev)
    position = i32([list(prompts)])
    for _ in range(steps):
        kept += 1
        x = torch.randn(n, hidden, generator=gen, device=dev).bfloat16()
        outputs.append(block(x, step, position, y).clone())
        position += 1
        lengths.append(kept.clone())
    return outputs, torch.stack(lengths)


if __name__ == "__main__":
    ys, lens = main()
    print("prompts of %d and %d tokens; %d steps; cached tokens at the end: %s" % (ys[0].shape[0], ys[1].shape[0], len(lens), lens[-1].tolist()))
    print("root mean square of the outputs: prompt %.4f, last step %.4f" % (ys[0].pow(2).mean().sqrt(), ys[-1].pow(2).mean().sqrt()))
