"""The attention blocks of an 8-bit decoder on the GPU, with a paged cache of keys and values in 4 bits, and the whole decoder around them.

A block is: norm of x + residual to 8-bit codes (the sum goes on as the next residual), the query-key-value product, norms of queries and
keys with the position rotation (which writes the cache in the same pass), attention, its output to codes, the output product. Whole prompts
attend to their own 16-bit keys and values; later tokens, one or several of each sequence at a time, to the cache.

``Sequences`` keeps the pages: which of them each sequence has, how long it is, and where its next tokens go. All layers' caches share them.

``python -m paper_2007_06919_gb300.attention`` runs prompts and greedy steps through a small random decoder.
"""
from __future__ import annotations

import torch

from . import aqd
from .feedforward import FeedForward, Head, _Part, _workspace


class Tokens:
    """Where a call's tokens lie: device tensors for the operators. starts [seqs + 1]: the tokens of each sequence; positions and slots [tokens];
    lengths [seqs]: places of each sequence with these tokens; table [seqs, columns]: its pages; fresh: whether all sequences begin here; one:
    whether each has one token. They may be dropped while a stream still reads them."""

    def __init__(self, starts, positions, slots, lengths, table, fresh: bool, one: bool):
        self.starts, self.positions, self.slots, self.lengths, self.table = starts, positions, slots, lengths, table
        self.fresh, self.one = fresh, one
        self._readers = set()

    def _read_on(self, stream):
        """Keeps the tensors' memory, once they are dropped, until this stream has finished with it."""
        handle = aqd._stream(stream)
        if handle not in self._readers:
            for t in (self.starts, self.positions, self.slots, self.lengths, self.table):
                t.record_stream(torch.cuda.current_stream() if stream is None else stream)
            self._readers.add(handle)


class Sequences:
    """Pages of the caches and the sequences that have them (host bookkeeping; `pages` pages of page_size places, tables of up to `columns` pages)."""

    def __init__(self, pages: int, page_size: int, columns: int, device="cuda"):
        self.page_size, self.columns, self.device = page_size, columns, device
        self.free = list(range(pages))
        self.pages: dict[int, list[int]] = {}
        self.lengths: dict[int, int] = {}

    def add(self, name: int):
        if name in self.pages:
            raise ValueError(f"sequence {name} is there already")
        self.pages[name], self.lengths[name] = [], 0

    def drop(self, name: int):
        """Its pages go to later sequences: calls that read them have to be on the streams that write them then, or done."""
        self.free += self.pages.pop(name)
        del self.lengths[name]

    def extend(self, names: list[int], counts: list[int]) -> Tokens:
        """Room for counts[i] more tokens of sequence names[i], in that order."""
        if len(names) != len(counts) or len(set(names)) != len(names) or any(n < 1 for n in counts):
            raise ValueError("one count of at least 1 for each of several different sequences")
        need = [-(-(self.lengths[s] + n) // self.page_size) for s, n in zip(names, counts)]
        if max(need, default=0) > self.columns or sum(need) - sum(len(self.pages[s]) for s in names) > len(self.free):
            raise ValueError("no room for these tokens")
        fresh = all(self.lengths[s] == 0 for s in names)
        starts, positions, slots, lengths, table = [0], [], [], [], []
        for s, n, pages in zip(names, counts, need):
            mine = self.pages[s]
            while len(mine) < pages:
                mine.append(self.free.pop())
            t = range(self.lengths[s], self.lengths[s] + n)
            positions += t
            slots += [mine[p // self.page_size] * self.page_size + p % self.page_size for p in t]
            starts.append(starts[-1] + n)
            self.lengths[s] += n
            lengths.append(self.lengths[s])
            table.append(mine + [-1] * (self.columns - len(mine)))

        def to(v, dtype):
            return torch.tensor(v, dtype=dtype, device=self.device)

        i32 = torch.int32
        return Tokens(to(starts, i32), to(positions, torch.int64), to(slots, torch.int64), to(lengths, i32),
                      to(table, i32).reshape(len(names), self.columns), fresh, all(n == 1 for n in counts))


class Attention(_Part):
    """One block: norm weight [d], qkv [(heads + 2 kv_heads) head_dim, d] (queries' rows, keys', values'), out [d, heads head_dim] in floating
    point, quantized here; q_norm and k_norm [head_dim] (None: no norm); inv_freq float32, a number for each pair that turns. Calls may come on several
    streams at a time, as a feed-forward block's; a cache is written by the calls that are given it."""

    def __init__(self, norm: torch.Tensor, qkv: torch.Tensor, out: torch.Tensor, *, heads: int, kv_heads: int, inv_freq: torch.Tensor,
                 q_norm: torch.Tensor | None = None, k_norm: torch.Tensor | None = None, eps: float = 1e-6, interleaved: bool = False):
        dim = out.shape[1] // heads
        if heads % kv_heads or out.shape[1] != heads * dim or qkv.shape != ((heads + 2 * kv_heads) * dim, out.shape[0]) or norm.shape != out.shape[:1]:
            raise ValueError("qkv must be [(heads + 2 kv_heads) head_dim, d], out [d, heads head_dim], norm [d]")
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dim
        self.norm, self.q_norm, self.k_norm, self.inv_freq, self.eps, self.interleaved = norm, q_norm, k_norm, inv_freq, eps, interleaved
        self.qkv = aqd.LinearWeights.from_float(qkv)
        self.out = aqd.LinearWeights.from_float(out)
        self._keep(norm, self.qkv, self.out)
        self._memory += [t for t in (q_norm, k_norm, inv_freq) if t is not None]

    def __call__(self, x: torch.Tensor, residual: torch.Tensor | None, tokens: Tokens, cache: aqd.KVCache, stream=None, workspace=None):
        """(block's output, x + residual) of x [tokens, d] in 16 bits, whose keys and values go into the cache. workspace: as a feed-forward block's."""
        if x.dtype not in (torch.float16, torch.bfloat16):
            raise ValueError(f"attention takes float16 or bfloat16, not {x.dtype}")
        if (cache.kv_heads, cache.head_dim) != (self.kv_heads, self.dim):
            raise ValueError("the cache has other heads than the block")
        self._read_on(stream)
        tokens._read_on(stream)
        if workspace is None:
            workspace = _workspace(x.shape[0], (self.qkv, self.out), stream)
        q8 = aqd.rms_norm_quant(x, self.norm, eps=self.eps, residual=residual, stream=stream)
        both = aqd.linear_int8(q8.codes, q8.scales, self.qkv, out_dtype=x.dtype, workspace=workspace, stream=stream)
        both = both.view(x.shape[0], self.heads + 2 * self.kv_heads, self.dim)
        q, k, v = both[:, :self.heads], both[:, self.heads:self.heads + self.kv_heads], both[:, self.heads + self.kv_heads:]
        # queries, and keys where a prompt needs them, in place: a row is read before it is written
        aqd.qk_norm_rope(q, k, tokens.positions, self.inv_freq, q_weight=self.q_norm, k_weight=self.k_norm, eps=self.eps, interleaved=self.interleaved,
                         q_out=q, k_out=k if tokens.fresh else None, v=v, cache=cache, slots=tokens.slots, stream=stream)
        if tokens.fresh:
            o = aqd.prompt_attention(q, k, v, tokens.starts, stream=stream)
        else:
            o = aqd.cache_attention(q, cache, tokens.table, tokens.lengths, starts=None if tokens.one else tokens.starts, stream=stream)
        h = aqd.quant_rows(o.view(x.shape[0], -1), stream=stream)
        y = aqd.linear_int8(h.codes, h.scales, self.out, out_dtype=x.dtype, workspace=workspace, stream=stream)
        return y, x if residual is None else q8.summed


class CausalDecoder:
    """Attention and feed-forward blocks in turn, and a head."""

    def __init__(self, blocks: list[tuple[Attention, FeedForward]], head: Head):
        self.blocks, self.head = blocks, head

    def caches(self, pages: int, page_size: int, device="cuda") -> list[aqd.KVCache]:
        """A cache for each layer."""
        return [aqd.KVCache(pages, page_size, a.kv_heads, a.dim, device) for a, _ in self.blocks]

    def __call__(self, x: torch.Tensor, tokens: Tokens, caches: list[aqd.KVCache], stream=None) -> torch.Tensor:
        """Logits [tokens, vocab] of tokens x [tokens, d] in 16 bits: whole prompts of new sequences, or further tokens of others. Types and caches that do
        not fit are refused before any cache is written."""
        if len(caches) != len(self.blocks) or any((c.kv_heads, c.head_dim) != (a.kv_heads, a.dim) for c, (a, _) in zip(caches, self.blocks)):
            raise ValueError("one cache for each layer, of its heads")
        layers = [w for a, f in self.blocks for w in (a.qkv, a.out, f.both, f.down)] + [self.head.proj]
        ws = _workspace(x.shape[0], layers, stream)
        residual = None
        for (attention, feed), cache in zip(self.blocks, caches):
            x, residual = attention(x, residual, tokens, cache, stream=stream, workspace=ws)
            x, residual = feed(x, residual, stream=stream, workspace=ws)
        return self.head(x, residual, stream=stream, workspace=ws)


def main():
    torch.manual_seed(0)
    d, hidden, vocab, heads, kv, dim = 512, 1024, 8192, 8, 2, 64

    def weight(n, k):
        return torch.randn(n, k, device="cuda") / k ** 0.5

    ones, head_ones = torch.ones(d, device="cuda", dtype=torch.bfloat16), torch.ones(dim, device="cuda", dtype=torch.bfloat16)
    inv_freq = 10000.0 ** (-torch.arange(0, dim, 2, device="cuda") / dim)
    net = CausalDecoder([(Attention(ones, weight((heads + 2 * kv) * dim, d), weight(d, heads * dim), heads=heads, kv_heads=kv, inv_freq=inv_freq, q_norm=head_ones, k_norm=head_ones),
                          FeedForward(ones, weight(hidden, d), weight(hidden, d), weight(d, hidden))) for _ in range(2)], Head(ones, 4 * weight(vocab, d)))
    embed = weight(vocab, d).bfloat16() * d ** 0.5
    sequences, caches = Sequences(64, 16, 16), net.caches(64, 16)
    prompts = [torch.randint(0, vocab, (n,), device="cuda") for n in (5, 40, 17)]
    for s in range(len(prompts)):
        sequences.add(s)
    where = sequences.extend([0, 1, 2], [len(p) for p in prompts])
    logits = net(embed[torch.cat(prompts)], where, caches)
    token = logits[where.starts[1:].long() - 1].argmax(1)
    for step in range(8):
        print(f"step {step}:", token.tolist())
        token = net(embed[token], sequences.extend([0, 1, 2], [1, 1, 1]), caches).argmax(1)


if __name__ == "__main__":
    main()
