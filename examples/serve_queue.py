"""A waiting queue served from the cache: match, prefill, decode, evict.

    python examples/serve_queue.py [--workload tiny] [--steps 8] [--keep 24]

What an engine does around this library, on one attention layer of a toy model (a token's q, k and v are rows of random
tables; the next token is the one that a random projection of the output picks):

  1. the K and V of earlier requests go into 8-bit pages, whole blocks, shared prefixes once (peek_kv_append);
  2. the queue is matched against the cache tree: h tokens of every prompt are there (peek_lpm_batch);
  3. the other tokens attend to the cached prefix and to themselves (peek_prefill_attention) and are appended;
  4. every request generates tokens, one step for all of them at a time, and collects the weight that falls on each of
     its blocks (peek_kv_append, peek_decode_attention);
  5. requests that hold more blocks than they may keep lose those of least weight (peek_kv_evict), their pages are free
     again unless another request shares them, and decoding goes on.
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import peek_workloads as W  # noqa: E402
from paper_2607_02525_amd import (KVPool, peek_decode_attention, peek_decode_attention_workspace,  # noqa: E402
                                  peek_kv_append, peek_kv_evict, peek_kv_evict_workspace, peek_prefill_attention,
                                  peek_prefill_attention_workspace)
from paper_2607_02525_amd.runner import HotPath  # noqa: E402


class Pages:
    """Which page holds what: free ones, users of each, the page of a cached block by the page before and its tokens."""

    def __init__(self, count: int):
        self.free = list(range(count - 1, -1, -1))
        self.users = np.zeros(count, np.int64)
        self.cached = {}

    def take(self, page: int | None = None) -> int:
        if page is None:
            if not self.free:
                raise RuntimeError("no free page")
            page = self.free.pop()
        self.users[page] += 1
        return page

    def drop(self, page: int):
        self.users[page] -= 1
        if self.users[page] == 0:
            self.free.append(page)


class Layer:
    """One attention layer of a toy model: q, k and v of a token by its id, and a next token for an output row."""

    def __init__(self, q_heads, kv_heads, dim, dtype, seed, rows=4096):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        make = lambda heads: torch.randn(rows, heads, dim, generator=gen, device="cuda").to(dtype)
        self.tables, self.rows = (make(q_heads), make(kv_heads), make(kv_heads)), rows
        self.head = torch.randn(q_heads * dim, rows, generator=gen, device="cuda").to(dtype)

    def qkv(self, tokens):
        return (t[tokens % self.rows] for t in self.tables)

    def next(self, out):
        return (out.reshape(out.shape[0], -1) @ self.head).argmax(1)


def _ints(values, dtype=torch.int32):
    return torch.as_tensor(np.asarray(values), dtype=dtype).cuda()


def _workspace(size):
    return torch.empty(max(size, 256), dtype=torch.uint8, device="cuda")


def fill_cache(pool, pages, layer, sequences, block):
    """Earlier requests' whole blocks into pages; a block that an earlier one has is shared."""
    tokens, offsets = sequences
    rows, context, new = [], [], []
    for s in range(len(offsets) - 1):
        seq = tokens[offsets[s]:offsets[s + 1]]
        whole, row, held = len(seq) // block, [], 0
        for b in range(whole):
            key = (row[-1] if row else -1, seq[b * block:(b + 1) * block].tobytes())
            if key in pages.cached:
                held = b + 1                 # what is cached of a sequence is a prefix of it
            else:
                pages.cached[key] = pages.take()
            row.append(pages.cached[key])
        rows.append(row)
        context.append(held * block)
        new.append(seq[held * block:whole * block])
    table = np.zeros((len(rows), max(1, max(map(len, rows)))), np.int32)
    for r, row in enumerate(rows):
        table[r, :len(row)] = row
    _, k, v = layer.qkv(_ints(np.concatenate(new), torch.int64))
    peek_kv_append(pool, k, v, _ints(np.cumsum([0] + [len(x) for x in new]), torch.int64), _ints(context), _ints(table))


def serve(workload, steps=8, keep=24, q_heads=8, kv_heads=2, dim=64, dtype=torch.bfloat16, format=torch.float8_e4m3fn,
          seed=0):
    """Serves the queue; returns what the last step saw and gave, for a look from outside."""
    w, B = workload, workload.block_size
    layer = Layer(q_heads, kv_heads, dim, dtype, seed)
    blocks = -(-(w.lengths + 2 * steps) // B)
    width = int(blocks.max())
    cached = np.diff(w.cache_sequences[1]) // B
    pages = Pages(int(blocks.sum() + cached.sum()))
    pool = KVPool.empty(len(pages.users), kv_heads, B, dim, dtype=format)
    fill_cache(pool, pages, layer, w.cache_sequences, B)

    # what of every prompt is cached
    hp = HotPath.from_sequences(*w.cache_sequences)
    hp.load_queue(w.tokens, w.offsets, B, w.threshold)
    hp.step()
    h = hp.results()["h"]
    table = np.zeros((w.n, width), np.int32)
    for r in range(w.n):
        prompt, page = w.prompt(r), -1
        for b in range(int(blocks[r])):
            page = pages.take(pages.cached[page, prompt[b * B:(b + 1) * B].tobytes()] if b < h[r] // B else None)
            table[r, b] = page

    # the prompts' other tokens, packed
    new = [w.prompt(r)[h[r]:] for r in range(w.n)]
    offsets, d_table, prefix = _ints(np.cumsum([0] + [len(x) for x in new]), torch.int64), _ints(table), _ints(h)
    q, k, v = layer.qkv(_ints(np.concatenate(new), torch.int64))
    out = torch.empty_like(q)
    ws = _workspace(peek_prefill_attention_workspace(w.n, q.shape[0], q_heads, kv_heads, dim, width * B))
    peek_prefill_attention(q, k, v, offsets, out, ws, pool=pool, prefix=prefix, block_table=d_table)
    peek_kv_append(pool, k, v, offsets, prefix, d_table)
    # (a prompt that is cached whole has no row; its first token is that of its id)
    token = _ints([w.prompt(r)[-1] for r in range(w.n)], torch.int64)
    if len(out) > 0:
        last = (offsets[1:] - 1).clamp(min=0)
        token = torch.where(offsets[1:] > offsets[:-1], layer.next(out[last]), token)

    context = _ints(w.lengths)
    one = torch.arange(w.n + 1, device="cuda")
    mass = torch.zeros(w.n, kv_heads, width, device="cuda")
    out, lse = torch.empty(w.n, q_heads, dim, dtype=dtype, device="cuda"), torch.empty(w.n, q_heads, device="cuda")
    ws = _workspace(peek_decode_attention_workspace(pool, w.n, q_heads, width, mass=True))

    def decode():
        nonlocal token, context, q
        q, k, v = layer.qkv(token)
        peek_kv_append(pool, k, v, one, context, d_table)
        context = context + 1
        peek_decode_attention(pool, q, context, d_table, out, ws, lse=lse, mass_in=mass, mass=mass)
        token = layer.next(out)

    for _ in range(steps):
        decode()
    gone = [torch.empty_like(context), torch.empty_like(d_table), torch.empty_like(mass), torch.empty_like(d_table),
            torch.empty_like(context)]
    peek_kv_evict(context, d_table, mass, torch.full_like(context, keep), B, 1, 2, *gone,
                  _workspace(peek_kv_evict_workspace(w.n, kv_heads, width)))
    context, d_table, mass, freed, num_freed = gone
    for row, count in zip(freed.cpu().numpy(), num_freed.cpu().numpy()):
        for page in row[:count]:
            pages.drop(int(page))
    for _ in range(steps):
        decode()
    return {"pool": pool, "q": q, "context": context, "table": d_table, "out": out, "lse": lse, "mass": mass, "h": h,
            "freed": num_freed, "free_pages": len(pages.free), "pages": len(pages.users)}


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--workload", default="tiny", choices=["tiny", "rag"])
    p.add_argument("--steps", type=int, default=8, help="tokens before, and after, the eviction")
    p.add_argument("--keep", type=int, default=24, help="blocks that a request may keep")
    a = p.parse_args()
    w = W.make(a.workload, 42) if a.workload == "tiny" else W.make_rag(42, n=256, n_cached=128)
    r = serve(w, a.steps, a.keep)
    print(f"{w.n} requests of {int(w.lengths.sum())} tokens, {int(r['h'].sum())} of them cached; {2 * a.steps} tokens "
          f"generated each; {int(r['freed'].sum())} blocks evicted, {r['free_pages']} of {r['pages']} pages free")


if __name__ == "__main__":
    main()
