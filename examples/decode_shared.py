"""Tokens for a queue whose prompts share long prefixes, with positions rotated into queries and keys.

    python examples/decode_shared.py [--workload rag] [--steps 8] [--keep 16]

The same toy layer as in serve_queue.py, its attention as a model with rotary positions runs it:

  1. earlier requests' queries and keys are normed and rotated, K and V go into pages (peek_rotate_append);
  2. the queue is matched, and the signals say which requests share a prefix (peek_lpm_batch, peek_queue_signals);
  3. the prompts' other tokens attend to the cached prefix and to themselves (peek_prefill_attention);
  4. the requests of a cluster whose tables begin with the same pages read these once a step
     (peek_shared_decode_attention);
  5. then every request looks at its `keep` most promising blocks only (peek_kv_bounds, peek_block_select,
     peek_sparse_decode_attention);
  6. the pages of the first request are read back as rows (peek_kv_read).
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import peek_workloads as W  # noqa: E402
from paper_2607_02525_amd import (PEEK_ROTARY_TURNS, KVPool, peek_block_select,  # noqa: E402
                                  peek_block_select_workspace, peek_kv_bounds, peek_kv_read, peek_prefill_attention,
                                  peek_prefill_attention_workspace, peek_rotary_frequencies, peek_rotate_append,
                                  peek_shared_decode_attention, peek_shared_decode_attention_workspace,
                                  peek_sparse_decode_attention, peek_sparse_decode_attention_workspace)
from paper_2607_02525_amd.runner import HotPath  # noqa: E402
from serve_queue import Layer, Pages, _ints, _workspace  # noqa: E402


def shared_groups(cluster_id, table, context, block):
    """members, group_offsets and shared for peek_shared_decode_attention: the clusters of the queue, with as many tokens
    as their members' tables begin with the same pages and all of them hold."""
    n = len(cluster_id)
    own = torch.arange(n, device=table.device)
    leader = torch.where(cluster_id >= 0, cluster_id.long(), own)
    _, members = torch.sort(leader, stable=True)
    leaders, sizes = torch.unique_consecutive(leader[members], return_counts=True)
    alike = (table == table[leader]).cumprod(1).sum(1) * block
    shared = torch.zeros(n, dtype=torch.long, device=table.device)
    shared = shared.scatter_reduce_(0, leader, torch.minimum(alike, context.long()), "amin", include_self=False)[leaders]
    offsets = torch.cat([torch.zeros(1, dtype=torch.long, device=table.device), sizes.cumsum(0)])
    return (x.to(torch.int32) for x in (members, offsets, torch.where(sizes > 1, shared, torch.zeros_like(shared))))


def generate(workload, steps=8, keep=16, q_heads=8, kv_heads=2, dim=64, dtype=torch.bfloat16,
             format=torch.float8_e4m3fn, seed=0):
    """Generates 2 * steps tokens for every request; returns what the last steps saw and gave, for a look from outside."""
    w, B = workload, workload.block_size
    layer = Layer(q_heads, kv_heads, dim, dtype, seed)
    blocks = -(-(w.lengths + 2 * steps) // B)
    width, sequences = int(blocks.max()), w.cache_sequences
    cached = np.diff(sequences[1]) // B
    pages = Pages(int(blocks.sum() + cached.sum()))
    pool = KVPool.empty(len(pages.users), kv_heads, B, dim, dtype=format)
    freq = torch.from_numpy(peek_rotary_frequencies(dim, 10000.0, PEEK_ROTARY_TURNS, 4.0, 2048.0)).cuda()
    gen = torch.Generator(device="cuda").manual_seed(seed)
    norms = dict(zip(("q_norm", "k_norm"), (1 + 0.1 * torch.randn(2, dim, generator=gen, device="cuda")).to(dtype)))

    def rotated(tokens, offsets, context, table, keys):
        """q of these tokens (and k, where asked for) as attention takes them; K and V are in the pages."""
        q, k, v = layer.qkv(tokens)
        peek_rotate_append(q, k, v, offsets, context, freq, q, k_out=k if keys else None, pool=pool, block_table=table,
                           **norms)
        return q, k, v

    # earlier requests' whole blocks, shared prefixes once
    rows, context, new = [], [], []
    for s in range(len(sequences[1]) - 1):
        seq, row, held = sequences[0][sequences[1][s]:sequences[1][s + 1]], [], 0
        for b in range(len(seq) // B):
            key = (row[-1] if row else -1, seq[b * B:(b + 1) * B].tobytes())
            if key in pages.cached:
                held = b + 1
            else:
                pages.cached[key] = pages.take()
            row.append(pages.cached[key])
        rows.append(row + [0] * (int(cached.max()) - len(row)))
        context.append(held * B)
        new.append(seq[held * B:len(row) * B])
    rotated(_ints(np.concatenate(new), torch.int64), _ints(np.cumsum([0] + [len(x) for x in new]), torch.int64),
            _ints(context), _ints(rows), False)

    # what of every prompt is cached, and who shares what
    hp = HotPath.from_sequences(*sequences)
    hp.load_queue(w.tokens, w.offsets, B, w.threshold)
    hp.step()
    found = hp.results()
    h, table = found["h"], np.zeros((w.n, width), np.int32)
    for r in range(w.n):
        prompt, page = w.prompt(r), -1
        for b in range(int(blocks[r])):
            page = pages.take(pages.cached[page, prompt[b * B:(b + 1) * B].tobytes()] if b < h[r] // B else None)
            table[r, b] = page
    table, prefix = _ints(table), _ints(h)

    # the prompts' other tokens, packed
    new = [w.prompt(r)[h[r]:] for r in range(w.n)]
    offsets = _ints(np.cumsum([0] + [len(x) for x in new]), torch.int64)
    token = _ints([w.prompt(r)[-1] for r in range(w.n)], torch.int64)
    if int(offsets[-1]) > 0:
        q, k, v = rotated(_ints(np.concatenate(new), torch.int64), offsets, prefix, table, True)
        out = torch.empty_like(q)
        ws = _workspace(peek_prefill_attention_workspace(w.n, len(q), q_heads, kv_heads, dim, width * B))
        peek_prefill_attention(q, k, v, offsets, out, ws, pool=pool, prefix=prefix, block_table=table)
        token = torch.where(offsets[1:] > offsets[:-1], layer.next(out[(offsets[1:] - 1).clamp(min=0)]), token)

    context = _ints(w.lengths)
    members, group_offsets, shared = shared_groups(_ints(found["cluster_id"]), table, context, B)
    one = torch.arange(w.n + 1, device="cuda")
    out, lse = torch.empty(w.n, q_heads, dim, dtype=dtype, device="cuda"), torch.empty(w.n, q_heads, device="cuda")
    ws = _workspace(max(peek_shared_decode_attention_workspace(pool, w.n, q_heads, width, len(shared)),
                        peek_block_select_workspace(pool, w.n, width),
                        peek_sparse_decode_attention_workspace(pool, w.n, q_heads, keep)))
    dense = {}
    for _ in range(steps):
        q = rotated(token, one, context, table, False)[0]
        context = context + 1
        peek_shared_decode_attention(pool, q, context, table, group_offsets, shared, out, ws, members=members, lse=lse)
        token = layer.next(out)
    dense.update(q=q, context=context, out=out.clone(), lse=lse.clone())

    bounds = torch.zeros(pool.num_pages, kv_heads, 2, dim, dtype=torch.int8, device="cuda")
    peek_kv_bounds(pool, None, context, table, bounds)
    kept = torch.empty(w.n, kv_heads, keep, dtype=torch.int32, device="cuda")
    tokens_kept = torch.empty(w.n, kv_heads, dtype=torch.int32, device="cuda")
    for _ in range(steps):
        q = rotated(token, one, context, table, False)[0]
        before, context = context, context + 1
        peek_kv_bounds(pool, before, context, table, bounds)
        peek_block_select(pool, bounds, q, context, table, 1, 2, tokens_kept, kept, ws)
        peek_sparse_decode_attention(pool, q, tokens_kept, kept, out, ws, lse=lse)
        token = layer.next(out)

    first = int(context[0])
    back = [torch.empty(first, kv_heads, dim, dtype=dtype, device="cuda") for _ in range(2)]
    peek_kv_read(pool, _ints([0, first], torch.int64), _ints([0]), table[:1], *back)
    return {"pool": pool, "table": table, "dense": dense, "shared": shared, "sizes": group_offsets.diff(), "q": q,
            "context": context, "kept": kept, "tokens_kept": tokens_kept, "out": out, "lse": lse, "back": back, "h": h}


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--workload", default="rag", choices=["tiny", "rag"])
    p.add_argument("--steps", type=int, default=8, help="tokens over all blocks, and over chosen ones")
    p.add_argument("--keep", type=int, default=16, help="blocks that a request looks at")
    a = p.parse_args()
    w = W.make(a.workload, 42) if a.workload == "tiny" else W.make_rag(42, n=256, n_cached=128)
    r = generate(w, a.steps, a.keep)
    tokens = int((r["shared"] * r["sizes"]).sum())
    print(f"{w.n} requests in {len(r['shared'])} groups, {tokens} of {int(r['dense']['context'].sum())} tokens read once "
          f"a group; then {int(r['tokens_kept'].sum()) // r['kept'].shape[1]} of {int(r['context'].sum())} tokens read")


if __name__ == "__main__":
    main()
