"""Beams over pages of latent rows: one worker's prefix cache with latent attention, random weights.

    python examples/latent_beams.py [--requests 8] [--beams 4] [--cache e4m3]

The resident chunks' latent rows are normed, rotated and written once (pp_rotary_write).  Prompts are
computed behind what is found of them, in pieces of `max_new` tokens: pp_block_tables places the new
tokens, pp_rotary_write rotates their queries and lays their rows into the pages, pp_latent_attention
reads them.  Behind its prompt a request goes on as `beams` rows, and each step every row takes up one
of its request's rows: pp_fork_tables shares the full pages, pp_page_copy copies the open ones, and
pp_free_pages finds what no row names any more, so nothing counts the sharers of a page.
"""

from __future__ import annotations

import argparse
import math
import os
import sys
import time
from dataclasses import dataclass

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from examples.prefix_cache import make_inputs  # noqa: E402
from paper_2608_01655_amd import binding as B  # noqa: E402

ROTARY = 64     # rotated elements of a row


@dataclass
class Layer:
    """Tokens to queries and latent rows; outputs from attention over them."""

    heads: int
    latent: int
    embed: torch.Tensor         # [vocabulary][width]
    query: torch.Tensor         # [width][heads (dim + ROTARY)]
    row: torch.Tensor           # [width][latent + ROTARY]
    norm: torch.Tensor          # [latent], of the rows' latent part
    key: torch.Tensor           # [heads][dim][latent]: expands a latent into a head's key, from the query's side
    value: torch.Tensor         # [heads][latent][dim]
    turns: torch.Tensor         # [ROTARY / 2]

    @staticmethod
    def random(heads=8, latent=256, dim=32, vocabulary=1024, width=256, dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=dtype)  # noqa: E731
        return Layer(heads, latent, rand(vocabulary, width), rand(width, heads * (dim + ROTARY)) / math.sqrt(width),
                     rand(width, latent + ROTARY) / math.sqrt(width), 1 + rand(latent) / 8,
                     rand(heads, dim, latent) / math.sqrt(latent), rand(heads, latent, dim) / math.sqrt(latent),
                     torch.from_numpy(B.pp_rotary_turns(ROTARY, 10000.0)).cuda())

    @property
    def scale(self):
        return 1 / math.sqrt(self.key.shape[1] + ROTARY)

    def rows(self, token):
        """Latent rows before norm and rotation, [t][1][latent + ROTARY]."""
        return (self.embed[token] @ self.row)[:, None]

    def queries(self, token):
        """Queries with the keys' expansion multiplied in, not yet rotated, [t][heads][latent + ROTARY]."""
        x = (self.embed[token] @ self.query).view(len(token), self.heads, -1)
        own, turning = x.split([self.key.shape[1], ROTARY], 2)
        return torch.cat([torch.bmm(own.transpose(0, 1).contiguous(), self.key).transpose(0, 1), turning], 2)

    def output(self, out):
        """[t][heads][dim] from attention's [t][heads][latent]."""
        return torch.bmm(out.transpose(0, 1).contiguous(), self.value).transpose(0, 1)


class Worker:
    """Pages of latent rows, and the rows of the block table that run."""

    def __init__(self, layer, parent, target, words, *, rows, max_len, page_size=16, cache=torch.bfloat16):
        """parent [n], words [n][chunk_tokens]: the tree and its chunks' tokens; target [n]: what stays here; rows: what
        runs at once."""
        self.layer, self.page, self.chunk, self.max_len = layer, page_size, words.shape[1], max_len
        d = self.device = torch.device("cuda")
        slot, _ = B.pp_cache_slots(target, int(target.sum()))
        self.n_slots = int(target.sum())
        self.resident = self.n_slots * (self.chunk // page_size)
        blocks = -(-max_len // page_size)
        pages = self.resident + (rows + 1) * blocks
        self.lines, self.slot = torch.from_numpy(B.pp_prefix_table(parent)).to(d), torch.from_numpy(slot).to(d)
        self.cache = torch.zeros((pages, 1, page_size, layer.latent + ROTARY), dtype=cache, device=d)
        # normed rows are some 4 at most
        self.k_scale = torch.full((1,), 1 / 16, device=d) if cache == torch.float8_e4m3fn else None
        i32 = dict(dtype=torch.int32, device=d)
        self.table, self.other = (torch.full((rows, blocks), -1, **i32) for _ in range(2))
        self.length = torch.zeros(0, **i32)
        self.free, self.count = torch.empty(pages, **i32), torch.empty(1, **i32)
        self.marks = torch.empty(pages, dtype=torch.uint8, device=d)
        node = torch.from_numpy((slot >= 0).nonzero()[0]).to(d)
        if len(node):
            i = torch.arange(self.chunk, device=d)
            position = (self.lines[node, 15:] * self.chunk + i).flatten().int()
            place = (self.slot[node].long()[:, None] * self.chunk + i).flatten()
            self.write(torch.as_tensor(words, device=d)[node].flatten(), position, place)

    def write(self, token, position, place, q=None):
        """Rows of tokens into the pages, and their queries rotated where they are."""
        layer = self.layer
        B.pp_rotary_write(position, layer.turns, q=q, q_out=q, q_first=layer.latent, k=layer.rows(token),
                          k_first=layer.latent, k_weight=layer.norm, slot_map=place, k_cache=self.cache,
                          k_scale=self.k_scale)

    def unnamed(self):
        """Pages that no running row names."""
        B.pp_free_pages(self.table[:len(self.length)], self.length, self.free, self.count, self.marks,
                        page_size=self.page, first=self.resident)
        return self.free[:int(self.count)]

    def step(self, leaf, tokens, cached, max_new):
        """One batch step.  leaf [R]; tokens [R]: every row's tokens so far; cached [R]: how many of them are done
        (-1: a new row).  Returns (out [t][heads][latent], query_start, start, end)."""
        R, d, layer = len(leaf), self.device, self.layer
        put = lambda x: torch.tensor(x, dtype=torch.int32, device=d)  # noqa: E731
        empty = lambda n, t=torch.int32: torch.empty(n, dtype=t, device=d)  # noqa: E731
        T = sum(min(max_new, len(t) - max(c, 0)) for t, c in zip(tokens, cached))   # at most
        self.length = put([max(c, 0) for c in cached])
        free = self.unnamed()
        query_start, start, end, taken = empty(R + 1), empty(R), empty(R), empty(1)
        slot_map, position = empty(T, torch.int64), empty(T)
        B.pp_block_tables(put(leaf), put([len(t) for t in tokens]), put(cached), self.lines, self.slot, free,
                          self.table[:R], query_start, start, end, slot_map, position, taken, page_size=self.page,
                          chunk_tokens=self.chunk, n_slots=self.n_slots, max_new=max_new)
        starts, ends = start.tolist(), end.tolist()
        if int(taken) > len(free):
            raise RuntimeError("out of pages")
        self.length = end
        new = torch.tensor([x for t, a, b in zip(tokens, starts, ends) for x in t[a:b]], device=d)
        t = len(new)
        q = layer.queries(new)
        self.write(new, position[:t], slot_map[:t], q)
        out = torch.empty((t, layer.heads, layer.latent), dtype=q.dtype, device=d)
        B.pp_latent_attention(q, self.cache, self.table[:R], query_start, end, out, scale=layer.scale,
                              max_new=max(b - a for a, b in zip(starts, ends)), max_len=max(ends),
                              k_scale=self.k_scale)
        return out, query_start.tolist(), starts, ends

    def fork(self, parent):
        """Row r goes on from row parent[r]: full pages are shared, open ones copied."""
        R, d = len(parent), self.device
        free = self.unnamed()
        length, source, target, count = torch.empty((4, R), dtype=torch.int32, device=d)
        taken = torch.empty(1, dtype=torch.int32, device=d)
        P = len(self.length)
        B.pp_fork_tables(torch.tensor(parent, dtype=torch.int32, device=d), self.length, self.table[:P], free,
                         self.other[:R], length, source, target, count, taken, page_size=self.page)
        if int(taken) > len(free):
            raise RuntimeError("out of pages")
        B.pp_page_copy([self.cache], source, target, count)
        self.table, self.other, self.length = self.other, self.table, length


def serve(worker, leaf, prompts, beams, decode, max_new, vocabulary=1024):
    """Serves all requests to `decode` tokens behind their prompts as `beams` rows each.  The next token and the row to
    go on from are read off a hash of the output's sign bits, which stands in for the rest of a model.  Returns
    (the rows' tokens, their last outputs [R beams][heads][latent], pages named at the end)."""
    R = len(leaf)
    tokens, cached = [list(map(int, p)) for p in prompts], [-1] * R
    weigh = torch.arange(1, worker.layer.output(torch.zeros((1, worker.layer.heads, worker.layer.latent), device="cuda",
                                                            dtype=worker.layer.value.dtype)).numel() + 1, device="cuda")

    def words(out):
        return ((worker.layer.output(out) > 0).flatten(1) * weigh).sum(1).tolist()

    last = [None] * R
    while any(c < len(t) for c, t in zip(cached, tokens)):
        out, begin, start, cached = worker.step(leaf, tokens, cached, max_new)
        for r in range(R):
            if cached[r] > start[r]:
                last[r] = out[begin[r + 1] - 1]
    rows = [r for r in range(R) for _ in range(beams)]       # the parents of the first fork
    leaf, last = [leaf[r] for r in rows], torch.stack(last)[rows]
    for n in range(decode):
        word = words(last)
        worker.fork(rows)
        tokens = [tokens[p] + [(w + 7 * r) % vocabulary] for r, (p, w) in enumerate(zip(rows, word))]
        last, _, _, _ = worker.step(leaf, tokens, [len(t) - 1 for t in tokens], 1)
        # rows of a request take up one another
        rows = [r // beams * beams + (w // 5 + r) % beams for r, w in enumerate(words(last))]
    worker.unnamed()
    return tokens, last, worker.cache.shape[0] - worker.resident - int(worker.count)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--requests", type=int, default=8)
    ap.add_argument("--beams", type=int, default=4)
    ap.add_argument("--decode", type=int, default=16)
    ap.add_argument("--max-new", type=int, default=256)
    ap.add_argument("--cache", choices=["bf16", "e4m3"], default="bf16")
    o = ap.parse_args()
    layer = Layer.random()
    parent, target, words, leaf, prompts = make_inputs(requests=o.requests)
    worker = Worker(layer, parent, target, words, rows=o.requests * o.beams, max_len=max(map(len, prompts)) + o.decode,
                    cache={"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}[o.cache])
    torch.cuda.synchronize()
    t = time.perf_counter()
    tokens, _, named = serve(worker, leaf, prompts, o.beams, o.decode, o.max_new)
    torch.cuda.synchronize()
    ms = (time.perf_counter() - t) * 1e3
    whole = sum(-(-len(t) // worker.page) for t in tokens)
    print(f"{o.requests} requests of {o.beams} rows over {int(target.sum())} resident chunks in {ms:.1f} ms: "
          f"{named} pages beside the chunks', {whole} where nothing is shared")


if __name__ == "__main__":
    main()
