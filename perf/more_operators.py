"""The cases on which the operators around a decode step over shared and long caches are measured.

A case is one pass of what an engine whose scheduler uses this library does between two tokens:

  rotate   the heads of q and k normed and rotated by their positions, K and V quantised into the
           pages in the same pass (peek_rotate_append); the touched blocks are read back
  read     tokens of the cache back as rows of 16 bits (peek_kv_read)
  shared   attention of one token per sequence where groups of sequences have their first pages in
           common, which are read once a group (peek_shared_decode_attention)
  bounds   the least and the largest key of every block, per head and element (peek_kv_bounds)
  sparse   a step over long contexts: the bounds of the newest block, the blocks whose bounds
           promise the most to each query (peek_block_select), attention over these
           (peek_sparse_decode_attention)

Lengths follow the queues of peek_workloads: chat (512 shared tokens, 64 to 512 of one's own), rag (a
cached prefix of a system prompt and a document), agentic (up to about 24000 tokens, and histories of
130000). Heads are generic: 8 key and value heads (2 to 16 in drawn cases), 1 to 16 query heads to
each, 64 or 128 numbers a head.

A cache is pages[P, 2, H, B, D] of 8-bit codes (K at 0, V at 1; B tokens to a block; float8 e4m3 or
int8) with scales[P, 2, H]; a value is its code times its scale. A sequence's tokens lie in the pages
that its row of the block table names, in order. Query head q reads key and value head q // group.
"""
import math
import random

import numpy as np
import torch

own = False

SCALE_MIN, SCALE_MAX = 2.0 ** -60, 2.0 ** 60
FORMATS = {"fp8": (torch.float8_e4m3fn, 448.0), "int8": (torch.int8, 127.0)}
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6


def listed():
    return [
        # one step of 64 running chats: every head of 64 tokens, K and V into their pages
        _rotate("rotate_step_64", 64, (1, 1), (576, 7000), heads=8, group=4, dim=128, block=16, dtype="bf16", fmt="fp8",
                rot=128, inter=False, norm=True, keys=False, stretch=1.0),
        # a batch of chat prompts after their hit; half of each head turns, neighbours in pairs
        _rotate("rotate_prompts_251", 251, (64, 512), (512, 512), heads=8, group=4, dim=128, block=16, dtype="f16",
                fmt="int8", rot=64, inter=True, norm=False, keys=True, stretch=1.0),
        # agents' next turns, far behind the trained length: frequencies stretched
        _rotate("rotate_agentic_40", 40, (200, 4000), (16000, 130000), heads=8, group=8, dim=128, block=16,
                dtype="bf16", fmt="fp8", rot=128, inter=False, norm=True, keys=True, stretch=8.0),
        # one user's document handed to another engine
        _read("read_one", 1, (5117, 5117), heads=8, dim=128, block=16, dtype="bf16", fmt="fp8"),
        # the cached documents of 64 questions
        _read("read_rag_64", 64, (3200, 7168), heads=8, dim=128, block=16, dtype="f16", fmt="int8"),
        # two users of one document: latency
        _shared("shared_pair_2", 2, 1, (5120, 5120), (45, 300), heads=8, group=5, dim=128, block=16, dtype="bf16",
                fmt="fp8"),
        # document chats, 1 to 20 users of each of 16 documents
        _shared("shared_rag_128", 128, 16, (3200, 7168), (32, 700), heads=8, group=4, dim=128, block=16, dtype="bf16",
                fmt="fp8"),
        # 192 agents that were forked from 4 histories
        _shared("shared_agentic_192", 192, 4, (12000, 16000), (500, 8000), heads=8, group=8, dim=128, block=64,
                dtype="f16", fmt="int8"),
        # the bounds of 64 cached documents
        _bounds("bounds_rag_64", 64, (0, 0), (3200, 7168), heads=8, dim=128, block=16, fmt="fp8"),
        # one agent's next token, an eighth of whose history is looked at: latency
        _sparse("sparse_one", 1, (23537, 23537), keep=184, heads=8, group=5, dim=128, block=16, dtype="bf16", fmt="fp8"),
        # a step of 64 agents
        _sparse("sparse_agentic_64", 64, (4000, 24000), keep=128, heads=8, group=4, dim=128, block=16, dtype="bf16",
                fmt="int8"),
        # a step over histories of up to 130000 tokens, blocks of 32
        _sparse("sparse_long_16", 16, (60000, 130000), keep=96, heads=8, group=8, dim=128, block=32, dtype="f16",
                fmt="fp8"),
    ]


def draw(rng):
    """Another case of these ranges, none dearer than the dearest listed one of its operator."""
    op = rng.choice(["rotate", "rotate", "read", "shared", "shared", "shared", "bounds", "sparse", "sparse", "sparse"])
    dim, dtype = rng.choice([64, 128, 128]), rng.choice(["bf16", "bf16", "f16"])
    heads, group = rng.choice([2, 4, 5, 8, 8, 10, 16]), rng.choice([1, 2, 4, 4, 5, 7, 8, 16])
    cache = {"heads": heads, "dim": dim, "block": rng.choice([4, 8, 16, 16, 32, 64, 128, 256]),
             "fmt": rng.choice(["fp8", "fp8", "int8"])}
    bound = max(_cost(c) for c in listed() if c["op"] == op)
    while True:
        n = _log_between(rng, 1, 256)
        if op == "rotate":
            new = rng.choice([1, 1, 7, 64, _log_between(rng, 1, 4000)])
            ctx = _log_between(rng, 1, 130000) if rng.random() < 0.8 else 0
            case = _rotate("", n, (max(1, new // 4), new), (ctx // 3, ctx), group=group, dtype=dtype,
                           rot=rng.choice([16, 32, 64, dim, dim, dim]), inter=rng.random() < 0.5,
                           norm=rng.random() < 0.6, keys=rng.random() < 0.5,
                           stretch=rng.choice([1.0, 1.0, 2.5, 8.0, 32.0]), **cache)
        elif op == "read":
            ctx = _log_between(rng, 1, 20000)
            case = _read("", n, (ctx // 4, ctx), dtype=dtype, **cache)
        elif op == "shared":
            hit, own_tokens = _log_between(rng, 16, 30000), _log_between(rng, 1, 8000)
            case = _shared("", n, rng.randint(1, max(1, n // 2)), (hit // 3, hit), (own_tokens // 8, own_tokens),
                           group=group, dtype=dtype, **cache)
        elif op == "bounds":
            ctx = _log_between(rng, 1, 30000)
            new = rng.choice([1, 64, ctx])
            case = _bounds("", n, (max(0, ctx - new) // 4,) * 2, (ctx // 4, ctx), **cache)
        else:
            ctx, keep = _log_between(rng, 1, 130000), _log_between(rng, 6, 500)
            case = _sparse("", n, (ctx // 4, ctx), keep=keep, group=group, dtype=dtype, **cache)
        if _cost(case) <= bound:
            break
    del case["name"]
    return case


def _log_between(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _case(name, op, n, **more):
    return {"name": name, "op": op, "n": n, **more}


def _rotate(name, n, new, ctx, heads, group, dim, block, dtype, fmt, rot, inter, norm, keys, stretch):
    return _case(name, "rotate", n, new_lo=new[0], new_hi=new[1], ctx_lo=ctx[0], ctx_hi=ctx[1], heads=heads, group=group,
                 dim=dim, block=block, dtype=dtype, fmt=fmt, rot=rot, inter=inter, norm=norm, keys=keys, stretch=stretch)


def _read(name, n, ctx, heads, dim, block, dtype, fmt):
    return _case(name, "read", n, ctx_lo=ctx[0], ctx_hi=ctx[1], heads=heads, dim=dim, block=block, dtype=dtype, fmt=fmt)


def _shared(name, n, groups, hit, new, heads, group, dim, block, dtype, fmt):
    return _case(name, "shared", n, groups=groups, hit_lo=hit[0], hit_hi=hit[1], new_lo=new[0], new_hi=new[1],
                 heads=heads, group=group, dim=dim, block=block, dtype=dtype, fmt=fmt)


def _bounds(name, n, first, ctx, heads, dim, block, fmt):
    return _case(name, "bounds", n, first_lo=first[0], first_hi=first[1], ctx_lo=ctx[0], ctx_hi=ctx[1], heads=heads,
                 dim=dim, block=block, fmt=fmt)


def _sparse(name, n, ctx, keep, heads, group, dim, block, dtype, fmt, sink=1, recent=2):
    return _case(name, "sparse", n, ctx_lo=ctx[0], ctx_hi=ctx[1], keep=keep, heads=heads, group=group, dim=dim,
                 block=block, dtype=dtype, fmt=fmt, sink=sink, recent=recent)


def _spread(case, key):
    """The case's lengths: the case's own, so that inputs of different seeds have one shape."""
    lo, hi, n = case[key + "_lo"], case[key + "_hi"], case["groups"] if key == "hit" else case["n"]
    rng = random.Random(f"{key} {lo} {hi} {n}")
    lens = [rng.randint(lo, hi) for _ in range(n)]
    lens[0] = hi
    if key == "hit":         # a hit is whole blocks
        lens = [x // case["block"] * case["block"] for x in lens]
    return lens


def _group_sizes(case):
    """n sequences in groups of uneven sizes, none empty."""
    n, groups = case["n"], case["groups"]
    rng = random.Random(f"groups {n} {groups}")
    cuts = sorted(rng.sample(range(1, n), groups - 1))
    return [b - a for a, b in zip([0] + cuts, cuts + [n])]


def _blocks(tokens, block):
    return -(-tokens // block)


def _cost(case):
    w = work(case)
    return w["bytes"] / 5e12 + w["flops"] / 1e15


def work(case):
    """What one pass cannot do without: inputs read once, outputs written once, and the products."""
    H, B, D, op = case["heads"], case["block"], case["dim"], case["op"]
    Hq = H * case.get("group", 1)
    if op == "rotate":
        new, ctx = _spread(case, "new"), _spread(case, "ctx")
        pages = sum(_blocks(c + t, B) - c // B for c, t in zip(ctx, new))
        held = sum(c % B for c in ctx)        # older tokens of the touched blocks, read back with the new ones
        rows = sum(new)
        return {"bytes": rows * D * (4 * Hq + 6 * H + (2 * H if case["keys"] else 0)) + (rows + held) * 2 * H * D * 3
                + pages * (2 * H * 4 + 4), "flops": rows * (Hq + H) * (3 * case["rot"] + (4 * D if case["norm"] else 0))}
    if op == "read":
        ctx = _spread(case, "ctx")
        return {"bytes": sum(ctx) * 2 * H * D * 3 + sum(_blocks(c, B) for c in ctx) * (2 * H * 4 + 4),
                "flops": sum(ctx) * 2 * H * D}
    if op == "shared":
        sizes, hit, new = _group_sizes(case), _spread(case, "hit"), _spread(case, "new")
        tokens = sum(hit) + sum(new)
        pages = sum(hit) // B + sum(_blocks(x, B) for x in new)
        pairs = sum(m * h for m, h in zip(sizes, hit)) + sum(new)
        return {"bytes": tokens * 2 * H * D + pages * (2 * H * 4 + 4) + case["n"] * Hq * (D * 4 + 4),
                "flops": 4 * D * Hq * pairs}
    ctx = _spread(case, "ctx")
    blocks = [_blocks(c, B) for c in ctx]
    if op == "bounds":
        first = _spread(case, "first")
        touched = sum(max(0, b - f // B) for b, f in zip(blocks, first))
        tokens = sum(max(0, c - f // B * B) for c, f in zip(ctx, first))
        return {"bytes": tokens * H * D + touched * (2 * H * D + 4 * H + 4), "flops": 2 * tokens * H * D}
    kept = [min(b, case["keep"]) for b in blocks]
    tokens = sum(min(c, k * B) for c, k in zip(ctx, kept))
    return {"bytes": sum(blocks) * (2 * H * D + 4 * H + 4) + tokens * 2 * H * D + sum(kept) * H * (2 * 4 + 8)
            + case["n"] * Hq * (D * 4 + 4), "flops": 4 * D * Hq * (sum(blocks) + tokens)}


# ---------------------------------------------------------------- inputs
def _pool(case, pages, gen, dev):
    """A cache in use: codes of normal values around means of the block's own, scales that differ from block to block."""
    dtype, most = FORMATS[case["fmt"]]
    shape = (pages, 2, case["heads"], case["block"], case["dim"])
    codes = torch.empty(shape, dtype=dtype, device=dev)
    step = max(1, (1 << 27) // max(1, codes[0].numel()))
    for p in range(0, pages, step):
        m = min(step, pages - p)
        x = torch.randn((m,) + shape[1:], generator=gen, device=dev, dtype=torch.float32)
        x += torch.randn((m, 2, shape[2], 1, shape[4]), generator=gen, device=dev, dtype=torch.float32)
        x = (x * (most / 6)).clamp_(-most, most)
        codes[p:p + step] = (x.round_() if case["fmt"] == "int8" else x).to(dtype)
    spread = torch.randint(0, 3, shape[:3], generator=gen, device=dev).float()
    scales = torch.exp2(spread - 1) * (4 / 512 if case["fmt"] == "fp8" else 4 / 127)
    return codes, scales.contiguous()


def _tables(case, lens, spare, gen, dev, first=None):
    """Block tables of these many tokens over shuffled pages; with `first`, only blocks from there on have pages."""
    B = case["block"]
    blocks = [_blocks(x, B) for x in lens]
    skip = [x // B for x in first] if first is not None else [0] * len(lens)
    width = max(1, max(blocks))
    pages = sum(b - s for b, s in zip(blocks, skip)) + spare
    ids = torch.randperm(pages, generator=gen, device=dev).to(torch.int32)
    rows = np.zeros((len(lens), width), np.int64)
    at = 0
    for r, (b, s) in enumerate(zip(blocks, skip)):
        rows[r, s:b] = np.arange(at, at + b - s)
        at += b - s
    return ids[torch.from_numpy(rows).to(dev)].contiguous(), pages


def _shared_tables(case, sizes, hit, new, gen, dev):
    """Rows of the sequences, group after group: a group's prefix first, then pages of the sequence's own."""
    B = case["block"]
    width = max(h // B + _blocks(x, B) for h, x in zip(np.repeat(hit, sizes).tolist(), new))
    rows = np.zeros((len(new), width), np.int64)
    at = r = 0
    for size, h in zip(sizes, hit):
        lead = np.arange(at, at + h // B)
        at += h // B
        for _ in range(size):
            mine = _blocks(new[r], B)
            rows[r, :h // B] = lead
            rows[r, h // B:h // B + mine] = np.arange(at, at + mine)
            at += mine
            r += 1
    ids = torch.randperm(at + 3, generator=gen, device=dev).to(torch.int32)
    return ids[torch.from_numpy(rows).to(dev)].contiguous(), at + 3


def _device_ints(values, dev, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device=dev)


def _offsets(lens, dev):
    return _device_ints(np.concatenate([[0], np.cumsum(lens)]).tolist(), dev, torch.int64)


def _frequencies(case, dev):
    """Radians a token of every pair; those of long waves slowed down where the context is stretched."""
    rot = case["rot"]
    f = 500000.0 ** (-np.arange(0, rot, 2, dtype=np.float64) / rot)
    if case["stretch"] > 1.0:
        turns = 8192 * f / (2 * math.pi)      # over the trained length
        keep = np.clip((turns - 1.0) / 3.0, 0.0, 1.0)
        f = f * (keep + (1 - keep) / case["stretch"])
    return torch.from_numpy(f).to(dev)


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    n, H, B, D, op = case["n"], case["heads"], case["block"], case["dim"], case["op"]
    Hq = H * case.get("group", 1)
    state = {"case": case}

    def normal(*shape, spread=1.0):
        x = torch.randn(shape, generator=gen, device=dev, dtype=torch.float32) * spread
        return x.to(TYPES[case["dtype"]])

    if op == "rotate":
        new, ctx = _spread(case, "new"), _spread(case, "ctx")
        state["table"], pages = _tables(case, [c + t for c, t in zip(ctx, new)], 3, gen, dev, first=ctx)
        state["pages"], state["scales"] = _pool(case, pages, gen, dev)
        # slices of a fused projection
        fused = normal(sum(new), Hq + 2 * H, D, spread=2.0)
        state["q"], state["k"], state["v"] = fused[:, :Hq], fused[:, Hq:Hq + H], fused[:, Hq + H:]
        state["offsets"], state["context"] = _offsets(new, dev), _device_ints(ctx, dev)
        state["freq"] = _frequencies(case, dev)
        state["magnitude"] = 1.0 if case["stretch"] == 1.0 else 0.1 * math.log(case["stretch"]) + 1.0
        if case["norm"]:
            state["q_norm"], state["k_norm"] = (1 + 0.2 * normal(D)).to(TYPES[case["dtype"]]), \
                (1 + 0.2 * normal(D)).to(TYPES[case["dtype"]])
        # the touched blocks, from their first token on
        state["first"] = _device_ints([c // B * B for c in ctx], dev)
        state["read_offsets"] = _offsets([c + t - c // B * B for c, t in zip(ctx, new)], dev)
        state["read_rows"] = sum(c + t - c // B * B for c, t in zip(ctx, new))
        state["q_out"] = torch.empty(sum(new), Hq, D, dtype=fused.dtype, device=dev)
        if case["keys"]:
            state["k_out"] = torch.empty(sum(new), H, D, dtype=fused.dtype, device=dev)
        state["k_read"] = torch.empty(state["read_rows"], H, D, dtype=fused.dtype, device=dev)
        state["v_read"] = torch.empty_like(state["k_read"])
    elif op == "read":
        ctx = _spread(case, "ctx")
        state["table"], pages = _tables(case, ctx, 3, gen, dev)
        state["pages"], state["scales"] = _pool(case, pages, gen, dev)
        state["first"], state["read_offsets"] = _device_ints([0] * n, dev), _offsets(ctx, dev)
        state["read_rows"] = sum(ctx)
        state["k_read"] = torch.empty(sum(ctx), H, D, dtype=TYPES[case["dtype"]], device=dev)
        state["v_read"] = torch.empty_like(state["k_read"])
    elif op == "shared":
        sizes, hit, new = _group_sizes(case), _spread(case, "hit"), _spread(case, "new")
        table, pages = _shared_tables(case, sizes, hit, new, gen, dev)
        # sequences in the order of their arrival, groups mixed; members names them group by group
        order = torch.from_numpy(np.random.default_rng(n).permutation(n)).to(dev)
        ctx = _device_ints([h + x for h, x in zip(np.repeat(hit, sizes).tolist(), new)], dev)
        state["table"], state["context"] = torch.empty_like(table), torch.empty_like(ctx)
        state["table"][order], state["context"][order] = table, ctx
        state["members"], state["group_offsets"] = order.to(torch.int32), _offsets(sizes, dev).to(torch.int32)
        state["shared"] = _device_ints(hit, dev)
        state["longest"] = max(h + x for h, x in zip(np.repeat(hit, sizes).tolist(), new))
        state["pages"], state["scales"] = _pool(case, pages, gen, dev)
        state["q"] = normal(n, Hq, D, spread=1.5)
        state["out"] = torch.empty_like(state["q"])
        state["lse"] = torch.empty(n, Hq, dtype=torch.float32, device=dev)
    else:
        ctx = _spread(case, "ctx")
        state["table"], pages = _tables(case, ctx, 3, gen, dev)
        state["pages"], state["scales"] = _pool(case, pages, gen, dev)
        state["context"] = _device_ints(ctx, dev)
        state["bounds"] = torch.zeros(pages, H, 2, D, dtype=torch.int8, device=dev)
        if op == "bounds":
            state["first"] = _device_ints(_spread(case, "first"), dev)
        else:
            # what earlier steps have left: bounds of all but the token that this step appended
            state["first"] = _device_ints([0] * n, dev)
            state["context"] -= 1
            _plain_bounds(state)
            state["context"] += 1
            state["first"] = state["context"] - 1
            keep = case["keep"]
            state["q"] = normal(n, Hq, D, spread=1.5)
            state["table_out"] = torch.empty(n, H, keep, dtype=torch.int32, device=dev)
            state["context_out"] = torch.empty(n, H, dtype=torch.int32, device=dev)
            state["out"] = torch.empty_like(state["q"])
            state["lse"] = torch.empty(n, Hq, dtype=torch.float32, device=dev)
    if own:
        import paper_2607_02525_amd as P
        state["pool"] = P.KVPool(state["pages"], state["scales"])
        width, size = state["table"].shape[1], 0
        if op == "shared":
            size = P.peek_shared_decode_attention_workspace(state["pool"], n, Hq, width, case["groups"])
        elif op == "sparse":
            size = max(P.peek_block_select_workspace(state["pool"], n, width),
                       P.peek_sparse_decode_attention_workspace(state["pool"], n, Hq, case["keep"]))
        state["workspace"] = torch.empty(max(size, 256), dtype=torch.uint8, device=dev)
    return state


def run(state):
    return (_run_own if own else _run_plain)[state["case"]["op"]](state)


# ---------------------------------------------------------------- the framework's operators
def _own_rotate(s):
    import paper_2607_02525_amd as P
    P.peek_rotate_append(s["q"], s["k"], s["v"], s["offsets"], s["context"], s["freq"], s["q_out"],
                         k_out=s.get("k_out"), pool=s["pool"], block_table=s["table"], interleaved=s["case"]["inter"],
                         magnitude=s["magnitude"], q_norm=s.get("q_norm"), k_norm=s.get("k_norm"), eps=EPS)
    out = _own_read(s)
    out["q"] = s["q_out"]
    if "k_out" in s:
        out["k"] = s["k_out"]
    return out


def _own_read(s):
    import paper_2607_02525_amd as P
    P.peek_kv_read(s["pool"], s["read_offsets"], s["first"], s["table"], s["k_read"], s["v_read"])
    return {"k_read": s["k_read"], "v_read": s["v_read"]}


def _own_shared(s):
    import paper_2607_02525_amd as P
    P.peek_shared_decode_attention(s["pool"], s["q"], s["context"], s["table"], s["group_offsets"], s["shared"],
                                   s["out"], s["workspace"], members=s["members"], lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_bounds(s):
    import paper_2607_02525_amd as P
    P.peek_kv_bounds(s["pool"], s["first"], s["context"], s["table"], s["bounds"])
    return {"bounds": s["bounds"]}


def _own_sparse(s):
    import paper_2607_02525_amd as P
    c = s["case"]
    P.peek_kv_bounds(s["pool"], s["first"], s["context"], s["table"], s["bounds"])
    P.peek_block_select(s["pool"], s["bounds"], s["q"], s["context"], s["table"], c["sink"], c["recent"],
                        s["context_out"], s["table_out"], s["workspace"])
    P.peek_sparse_decode_attention(s["pool"], s["q"], s["context_out"], s["table_out"], s["out"], s["workspace"],
                                   lse=s["lse"])
    return {"bounds": s["bounds"], "context": s["context_out"], "table": s["table_out"], "out": s["out"],
            "lse": s["lse"]}


_run_own = {"rotate": _own_rotate, "read": _own_read, "shared": _own_shared, "bounds": _own_bounds,
            "sparse": _own_sparse}


# ---------------------------------------------------------------- plain forms, 32 bits
def _scale_of(amax, fmt):
    """fp8: the smallest power of two under which amax is no larger than 448. int8: amax / 127."""
    if fmt == "int8":
        return (amax * np.float32(1.0 / 127.0)).clamp(SCALE_MIN, SCALE_MAX)
    m, e = torch.frexp(amax)
    e = torch.where(m <= 0.875, e - 9, e - 8)
    e = torch.where(amax > 0, e, torch.full_like(e, -60)).clamp(-60, 60)
    return torch.ldexp(torch.ones_like(amax), e)


def _codes_of(x, scale, fmt):
    dtype, most = FORMATS[fmt]
    x = (x / scale).clamp(-most, most)
    return (x.round() if fmt == "int8" else x).to(dtype)


def _values(codes, scales):
    return codes.to(torch.float32) * scales[..., None, None]


def _rows_of(offsets, total):
    """The sequence of every row, and the row's number in it."""
    at = torch.arange(total, device=offsets.device)
    row = torch.searchsorted(offsets, at, right=True) - 1
    return row, at - offsets[row]


def _rotated(x, norm, cos, sin, inter):
    """Heads [rows, heads, D], normed and turned by [rows, rot / 2] angles."""
    x = x.float()
    if norm is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * norm.float()
    cos, sin, rot = cos[:, None], sin[:, None], 2 * cos.shape[1]
    t = x[..., :rot]
    a, b = (t[..., 0::2], t[..., 1::2]) if inter else (t[..., :rot // 2], t[..., rot // 2:])
    u, w = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([u, w], -1).flatten(-2) if inter else torch.cat([u, w], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain_rotate(s):
    c, B = s["case"], s["case"]["block"]
    total, dev = s["q"].shape[0], s["q"].device
    row, i = _rows_of(s["offsets"], total)
    pos = s["context"][row].long() + i
    angle = pos.double()[:, None] * s["freq"]
    cos, sin = (torch.cos(angle) * s["magnitude"]).float(), (torch.sin(angle) * s["magnitude"]).float()
    q = _rotated(s["q"], s.get("q_norm"), cos, sin, c["inter"]).to(s["q"].dtype)
    k = _rotated(s["k"], s.get("k_norm"), cos, sin, c["inter"]).to(s["q"].dtype)
    # into the pages: the rows as they are in 16 bits
    codes, scales, P = s["pages"], s["scales"], s["pages"].shape[0]
    x = torch.stack([k, s["v"]], 1).float()                               # [total, 2, H, D]
    page, slot = s["table"][row, pos // B].long(), pos % B
    amax = torch.zeros(P, 2, c["heads"], device=dev).index_reduce_(0, page, x.abs().amax(-1), "amax")
    written = torch.zeros(P, dtype=torch.bool, device=dev).index_fill_(0, page, True)
    # older tokens of a block: those before its first new one
    begin = torch.full((P,), B, device=dev, dtype=torch.int64).index_reduce_(0, page, slot, "amin")
    new = _scale_of(amax, c["fmt"])
    has_old = written & (begin > 0)
    new = torch.where(has_old[:, None, None], torch.maximum(new, scales), new)
    again = has_old[:, None, None] & (new > scales)
    old = torch.arange(B, device=dev)[None] < begin[:, None]
    again = again[..., None, None] & old[:, None, None, :, None]
    requant = _codes_of(codes.float() * scales[..., None, None], new[..., None, None], c["fmt"])
    raw, fresh = codes.view(torch.uint8), requant.view(torch.uint8)
    raw.copy_(torch.where(again, fresh, raw))
    scales.copy_(torch.where(written[:, None, None], new, scales))
    raw[page, :, :, slot] = _codes_of(x, scales[page][..., None], c["fmt"]).view(torch.uint8)
    out = _plain_read(s)
    out["q"] = q
    if c["keys"]:
        out["k"] = k
    return out


def _plain_read(s):
    c, B = s["case"], s["case"]["block"]
    row, i = _rows_of(s["read_offsets"], s["read_rows"])
    pos = s["first"][row].long() + i
    page, slot = s["table"][row, pos // B].long(), pos % B
    codes = s["pages"].view(torch.uint8)[page, :, :, slot].view(s["pages"].dtype)        # [rows, 2, H, D]
    x = (codes.float() * s["scales"][page][..., None]).to(TYPES[c["dtype"]])
    return {"k_read": x[:, 0].contiguous(), "v_read": x[:, 1].contiguous()}


def _attend(q, keys, values, live):
    """q [n, H, G, D] over keys, values [n, H, L, D], of which live [n, H or 1, L] are there: rows of 0 without any."""
    logits = torch.matmul(q, keys.transpose(2, 3).contiguous()) * (q.shape[-1] ** -0.5)
    logits = logits.masked_fill_(~live[:, :, None], -math.inf)
    top = logits.amax(-1, keepdim=True).clamp_(min=torch.finfo(logits.dtype).min)
    p = torch.exp(logits - top)
    total = p.sum(-1, keepdim=True)
    lse = (top + total.log())[..., 0]
    return torch.matmul(p, values) / total.clamp(min=torch.finfo(total.dtype).tiny), lse


def _plain_shared(s):
    c = s["case"]
    n, H, G, D, B = c["n"], c["heads"], c["group"], c["dim"], c["block"]
    ids = s["table"].long()
    live = torch.arange(ids.shape[1] * B, device=ids.device)[None, None] < s["context"][:, None, None]
    codes = s["pages"].view(torch.uint8)
    keys, values = (_values(codes[ids, i].view(s["pages"].dtype), s["scales"][ids, i])
                    .transpose(1, 2).reshape(n, H, -1, D) for i in (0, 1))
    out, lse = _attend(s["q"].float().view(n, H, G, D), keys, values, live)
    return {"out": out.view(n, H * G, D).to(s["q"].dtype), "lse": lse.reshape(n, H * G)}


def _plain_bounds(s):
    """Largest and smallest key code of every block from `first` on; of float8, in steps of 4, rounded outwards."""
    B, table, bounds = s["case"]["block"], s["table"], s["bounds"]
    at = torch.arange(table.shape[1], device=table.device)[None]
    row, b = torch.nonzero((at >= (s["first"] // B)[:, None]) & (at * B < s["context"][:, None]), as_tuple=True)
    page = table[row, b].long()
    held = torch.arange(B, device=table.device)[None] + (b * B)[:, None] < s["context"][row][:, None]
    held = held[:, None, :, None]                                                        # [blocks, 1, B, 1]
    x = s["pages"].view(torch.uint8)[page, 0].view(s["pages"].dtype).float()             # [blocks, H, B, D]
    hi = x.masked_fill(~held, -math.inf).amax(2)
    lo = x.masked_fill(~held, math.inf).amin(2)
    if s["pages"].dtype != torch.int8:
        hi, lo = torch.ceil(hi / 4), torch.floor(lo / 4)
    bounds[page] = torch.stack([hi, lo], 2).clamp(-127, 127).to(torch.int8)
    return {"bounds": bounds}


def _plain_sparse(s):
    c = s["case"]
    n, H, G, D, B, K = c["n"], c["heads"], c["group"], c["dim"], c["block"], c["keep"]
    bounds = _plain_bounds(s)["bounds"]
    table, ctx, dev = s["table"], s["context"], s["table"].device
    W = table.shape[1]
    # queries to whole numbers of up to 127, by a power of two
    q = s["q"].float().view(n, H, G, D)
    e = torch.frexp(q.abs().amax(-1, keepdim=True))[1] - 7
    code = torch.ldexp(q, -e).round().clamp(-127, 127)
    # sums of whole numbers below 2^23: exact in 32 bits in any order
    x = bounds[table.long()].float().permute(0, 2, 3, 4, 1)                              # [n, H, 2, D, W]
    dot = torch.matmul(code.clamp(min=0), x[:, :, 0].contiguous()) + torch.matmul(code.clamp(max=0), x[:, :, 1].contiguous())
    step = s["scales"][table.long(), 0].transpose(1, 2) * (1.0 if c["fmt"] == "int8" else 4.0)
    score = torch.ldexp(dot, e).amax(2) * step                                           # [n, H, W]
    nb = (ctx + B - 1) // B
    at = torch.arange(W, device=dev)[None]
    must = (at < c["sink"]) | (at >= (nb - c["recent"])[:, None])
    score = score.masked_fill(must[:, None], math.inf).masked_fill((at >= nb[:, None])[:, None], -math.inf)
    best = torch.sort(score, dim=-1, descending=True, stable=True)[1][..., :K]
    if W < K:
        best = torch.cat([best, torch.full((n, H, K - W), W, device=dev)], -1)
    best = torch.sort(torch.where(best < nb[:, None, None], best, torch.full_like(best, 1 << 30)), dim=-1)[0]
    live = best < (1 << 30)
    blocks = torch.where(live, best, torch.zeros_like(best))
    rows = torch.arange(n, device=dev)[:, None, None]
    table_out = torch.where(live, table[rows, blocks], torch.full_like(table[rows, blocks], -1))
    kept = live.sum(-1)
    context_out = (kept * B - (nb * B - ctx)[:, None]).clamp(min=0).to(torch.int32)
    page = torch.where(live, table_out, torch.zeros_like(table_out)).long()
    heads = torch.arange(H, device=dev)[None, :, None]
    raw = s["pages"].view(torch.uint8)
    keys, values = (_values(raw[page, i, heads].view(s["pages"].dtype), s["scales"][page, i, heads])
                    .reshape(n, H, K * B, D) for i in (0, 1))
    seen = torch.arange(K * B, device=dev)[None, None] < context_out[..., None]
    out, lse = _attend(q, keys, values, seen)
    return {"bounds": bounds, "context": context_out, "table": table_out, "out": out.view(n, H * G, D).to(s["q"].dtype),
            "lse": lse.reshape(n, H * G)}


_run_plain = {"rotate": _plain_rotate, "read": _plain_read, "shared": _plain_shared, "bounds": _plain_bounds,
              "sparse": _plain_sparse}


# ---------------------------------------------------------------- from the definitions, 64 bits
def _exact_softmax(q, keys, values):
    """q [H, G, D], keys, values [H, S, D], all float64: the attention's rows [H * G, D] and their logarithms."""
    H, G, D = q.shape
    x = (q[:, :, None, :] * (D ** -0.5)) @ keys.transpose(1, 2).contiguous()[:, None]
    x = x[:, :, 0]
    lse = torch.logsumexp(x, -1)
    return (torch.exp(x - lse[..., None]) @ values).reshape(H * G, D), lse.reshape(-1)


def _exact_tokens(s, ids, tokens):
    """K and V [H, tokens, D] in 64 bits of the pages in `ids`."""
    x = s["pages"].view(torch.uint8)[ids].view(s["pages"].dtype).to(torch.float32).double() * s["scales"][ids].double()[..., None, None]
    x = x.permute(1, 2, 0, 3, 4).flatten(2, 3)[:, :, :tokens]
    return x[0].contiguous(), x[1].contiguous()


def exact(case, seed):
    if case["op"] == "bounds":       # whole numbers
        return None
    s = prepare(case, seed)
    op, n, H, B, D = case["op"], case["n"], case["heads"], case["block"], case["dim"]
    G = case.get("group", 1)
    if op == "read":
        k, v = [], []
        for r, t in enumerate(_spread(case, "ctx")):
            a, b = _exact_tokens(s, s["table"][r, :_blocks(t, B)].long(), t)
            k.append(a.transpose(0, 1))
            v.append(b.transpose(0, 1))
        return {"k_read": torch.cat(k), "v_read": torch.cat(v)}
    if op == "rotate":
        pos = torch.cat([torch.arange(c, c + t, device=s["q"].device) for c, t in zip(_spread(case, "ctx"), _spread(case, "new"))])
        turn = torch.polar(torch.full((len(pos), case["rot"] // 2), s["magnitude"], dtype=torch.float64, device=pos.device),
                           pos.double()[:, None] * s["freq"])[:, None]

        def heads(x, weight):
            x = x.double()
            if weight is not None:
                x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.double()
            head, tail = x[..., :case["rot"]], x[..., case["rot"]:]
            pairs = head.unflatten(-1, (-1, 2)) if case["inter"] else head.unflatten(-1, (2, -1)).transpose(-1, -2)
            z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
            z = z if case["inter"] else z.transpose(-1, -2)
            return torch.cat([z.flatten(-2), tail], -1)

        out = {"k_read": None, "v_read": None, "q": heads(s["q"], s.get("q_norm"))}
        if case["keys"]:
            out["k"] = heads(s["k"], s.get("k_norm"))
        return out
    out = torch.zeros(n, H * G, D, dtype=torch.float64, device=s["q"].device)
    lse = torch.full((n, H * G), -math.inf, dtype=torch.float64, device=s["q"].device)
    q = s["q"].double().view(n, H, G, D)
    if op == "shared":
        for r, t in enumerate(s["context"].tolist()):
            if t > 0:
                out[r], lse[r] = _exact_softmax(q[r], *_exact_tokens(s, s["table"][r, :_blocks(t, B)].long(), t))
        return {"out": out, "lse": lse}
    picked = _exact_blocks(s)
    for r in range(n):
        for h in range(H):
            chosen = picked[r][h]
            if chosen:
                t = len(chosen) * B - (-int(s["context"][r]) % B)
                ids = s["table"][r, torch.tensor(chosen, device=q.device)].long()
                k, v = _exact_tokens({"pages": s["pages"][:, :, h:h + 1], "scales": s["scales"][:, :, h:h + 1]}, ids, t)
                out[r, h * G:(h + 1) * G], lse[r, h * G:(h + 1) * G] = _exact_softmax(q[r, h:h + 1], k, v)
    return {"bounds": None, "context": None, "table": None, "out": out, "lse": lse}


def _exact_blocks(s):
    """The kept blocks of every sequence and head, in whole numbers on the host."""
    c = s["case"]
    B, H, G, K = c["block"], c["heads"], c["group"], c["keep"]
    picked = []
    for r, t in enumerate(s["context"].tolist()):
        nb = _blocks(t, B)
        ids = s["table"][r, :nb].long()
        codes = s["pages"].view(torch.uint8)[ids, 0].view(s["pages"].dtype).to(torch.float32).double()      # [nb, H, B, D]
        last = codes[-1:, :, :t - (nb - 1) * B]
        hi = torch.cat([codes[:-1].amax(2), last.amax(2)])
        lo = torch.cat([codes[:-1].amin(2), last.amin(2)])
        step = 1
        if c["fmt"] != "int8":
            step, hi, lo = 4, (hi / 4).ceil(), (lo / 4).floor()
        hi, lo = hi.clamp(-127, 127), lo.clamp(-127, 127)
        q = s["q"][r].double().view(H, G, -1)
        unit = torch.exp2(torch.floor(torch.log2(q.abs().amax(-1, keepdim=True))) - 6)
        w = (q / unit).round().clamp(-127, 127)
        best = torch.full((nb, H), -math.inf, dtype=torch.float64, device=q.device)
        for g in range(G):
            dot = torch.maximum(w[None, :, g] * hi, w[None, :, g] * lo).sum(-1) * unit[None, :, g, 0]
            best = torch.maximum(best, dot)
        # (the product with the block's scale is a 32-bit number: equal scores are ties)
        score = (best.float() * (s["scales"][ids, 0] * step)).cpu().numpy()
        picked.append([])
        for h in range(H):
            must = [b for b in range(nb) if b < c["sink"] or b >= nb - c["recent"]]
            rest = [b for b in np.argsort(-score[:, h], kind="stable").tolist() if c["sink"] <= b < nb - c["recent"]]
            picked[-1].append(sorted(must + rest[:max(0, K - len(must))]))
    return picked
