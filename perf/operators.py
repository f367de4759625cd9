"""The cases on which the attention operators of this framework are measured.

A case is one call of one operator, at the sizes of an engine whose scheduler uses this library:

  append   K and V of new tokens into the 8-bit pages of the cache (peek_kv_append)
  prefill  causal attention of packed prompts: the cached prefix that the match found, read from
           the pages, and the prompt's own tokens after it (peek_prefill_attention)
  decode   attention of one new token per sequence over its cached pages, with or without the
           weight that falls on every block (peek_decode_attention)
  evict    the blocks of least accumulated weight leave their sequences' tables (peek_kv_evict)

Lengths follow the queues of peek_workloads: chat (512 shared tokens, 64 to 512 of one's own), rag
(a cached prefix of a system prompt and a document, 32 to 256 tokens of query), agentic (up to
about 24000 tokens), nosharing (512 to 4096 tokens, nothing cached). Heads are generic: 8 key and
value heads (2 to 16 in drawn cases), 1 to 16 query heads to each, 64 or 128 numbers a head.

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


def listed():
    return [
        # one step of 64 running chats: each appends the token it has just computed
        _append("append_tokens_64", 64, (1, 1), (576, 7000), heads=8, dim=128, block=16, dtype="bf16", fmt="fp8"),
        # K and V of a batch of chat prompts after their hit, into int8 pages
        _append("append_prompts_251", 251, (64, 512), (512, 512), heads=8, dim=128, block=16, dtype="f16", fmt="int8"),
        # a single short prompt on an idle engine, nothing cached: latency
        _prefill("prefill_one_short", 1, (45, 45), (0, 0), heads=8, group=4, dim=128, block=16, dtype="bf16", fmt="fp8"),
        # the 64-prompt chat queue, 512 tokens of each found in the cache
        _prefill("prefill_chat_64", 64, (64, 512), (512, 512), heads=8, group=4, dim=128, block=16, dtype="bf16",
                 fmt="fp8"),
        # document questions: short queries after long cached prefixes
        _prefill("prefill_rag_64", 64, (32, 256), (3200, 7168), heads=8, group=5, dim=128, block=16, dtype="bf16",
                 fmt="int8"),
        # cold agent histories, prompts of very different lengths
        _prefill("prefill_agentic_cold_5", 5, (900, 24000), (0, 0), heads=8, group=4, dim=128, block=16, dtype="bf16",
                 fmt="fp8"),
        # one agent's next turn: few rows against a long cached prefix, small heads
        _prefill("prefill_turn_1", 1, (37, 37), (23552, 23552), heads=8, group=8, dim=64, block=32, dtype="f16",
                 fmt="fp8"),
        # one user's next token after a document: latency
        _decode("decode_one", 1, (5117, 5117), heads=8, group=5, dim=128, block=16, dtype="bf16", fmt="fp8"),
        # a step of 64 document chats that also weighs the blocks for eviction
        _decode("decode_rag_weights_64", 64, (1100, 7400), heads=8, group=4, dim=128, block=16, dtype="bf16", fmt="fp8",
                mass=True),
        # the largest step: 192 agents with long histories, int8, blocks of 64 tokens
        _decode("decode_agentic_192", 192, (2000, 24000), heads=8, group=8, dim=128, block=64, dtype="f16", fmt="int8"),
        # halving the caches of 64 document chats
        _evict("evict_rag_64", 64, (1100, 7400), heads=8, block=16, keep=0.5),
        # bounding the caches of 192 agents, some of them very long
        _evict("evict_agentic_192", 192, (4000, 130000), heads=8, block=16, keep=0.75),
    ]


def draw(rng):
    """Another case of these ranges, none dearer than the largest listed one of its operator."""
    op = rng.choice(["append", "prefill", "prefill", "decode", "decode", "evict"])
    heads = rng.choice([2, 4, 5, 8, 8, 10, 16])
    group = rng.choice([1, 2, 4, 4, 5, 7, 8, 16])
    shape = {"heads": heads, "dim": rng.choice([64, 128, 128]),
             "block": rng.choice([4, 8, 16, 16, 32, 64, 128, 256]), "dtype": rng.choice(["bf16", "bf16", "f16"]),
             "fmt": rng.choice(["fp8", "fp8", "int8"])}
    bound = max(_cost(c) for c in listed() if c["op"] == op)
    while True:
        n = _log_between(rng, 1, 256)
        if op == "append":
            ctx = _log_between(rng, 1, 8000) if rng.random() < 0.8 else 0
            new = rng.choice([1, 1, 7, 64, _log_between(rng, 1, 2000)])
            case = _append("", n, (max(1, new // 4), new), (ctx // 3, ctx), **shape)
        elif op == "prefill":
            new, hit = _log_between(rng, 1, 16000), rng.choice([0, 1, 1]) * _log_between(rng, 16, 16000)
            case = _prefill("", n, (max(1, new // 5), new), (hit // 3, hit), group=group, **shape)
        elif op == "decode":
            ctx = _log_between(rng, 1, 30000)
            case = _decode("", n, (ctx // 8, ctx), group=group, mass=rng.random() < 0.4, **shape)
        else:
            ctx = _log_between(rng, 1, 130000)
            case = _evict("", n, (ctx // 8, ctx), heads=heads, block=shape["block"],
                          keep=rng.choice([0.1, 0.5, 0.75, 0.9]))
        if _cost(case) <= bound:
            break
    del case["name"]
    return case


def _log_between(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _case(name, op, n, **more):
    return {"name": name, "op": op, "n": n, **more}


def _append(name, n, new, ctx, heads, dim, block, dtype, fmt):
    return _case(name, "append", n, new_lo=new[0], new_hi=new[1], ctx_lo=ctx[0], ctx_hi=ctx[1], heads=heads, dim=dim,
                 block=block, dtype=dtype, fmt=fmt)


def _prefill(name, n, new, hit, heads, group, dim, block, dtype, fmt):
    return _case(name, "prefill", n, new_lo=new[0], new_hi=new[1], hit_lo=hit[0], hit_hi=hit[1], heads=heads,
                 group=group, dim=dim, block=block, dtype=dtype, fmt=fmt)


def _decode(name, n, ctx, heads, group, dim, block, dtype, fmt, mass=False):
    return _case(name, "decode", n, ctx_lo=ctx[0], ctx_hi=ctx[1], heads=heads, group=group, dim=dim, block=block,
                 dtype=dtype, fmt=fmt, mass=mass)


def _evict(name, n, ctx, heads, block, keep, sink=1, recent=4):
    return _case(name, "evict", n, ctx_lo=ctx[0], ctx_hi=ctx[1], heads=heads, block=block, keep=keep, sink=sink,
                 recent=recent)


def _spread(case, key):
    """The case's lengths: the case's own, so that inputs of different seeds have one shape."""
    lo, hi, n = case[key + "_lo"], case[key + "_hi"], case["n"]
    rng = random.Random(f"{key} {lo} {hi} {n}")
    lens = [rng.randint(lo, hi) for _ in range(n)]
    lens[0] = hi
    if key == "hit":         # a hit is whole blocks
        lens = [x // case["block"] * case["block"] for x in lens]
    return lens


def _blocks(tokens, block):
    return -(-tokens // block)


def _cost(case):
    w = work(case)
    return w["bytes"] / 5e12 + w["flops"] / 1e15


def work(case):
    """What one pass cannot do without: inputs read once, outputs written once, and the products."""
    H, B = case["heads"], case["block"]
    if case["op"] == "append":
        new, ctx, D = _spread(case, "new"), _spread(case, "ctx"), case["dim"]
        pages = sum(_blocks(c + t, B) - c // B for c, t in zip(ctx, new))
        return {"bytes": sum(new) * 2 * H * D * 3 + pages * (2 * H * 4 + 4), "flops": 4 * sum(new) * H * D}
    if case["op"] == "prefill":
        new, hit, D, Hq = _spread(case, "new"), _spread(case, "hit"), case["dim"], case["heads"] * case["group"]
        pairs = sum(t * h + t * (t + 1) // 2 for t, h in zip(new, hit))
        rows = sum(new)
        return {"bytes": rows * D * 2 * (2 * Hq + 2 * H) + sum(hit) * 2 * H * D + sum(hit) // B * (2 * H * 4 + 4)
                + rows * Hq * 4, "flops": 4 * D * Hq * pairs}
    if case["op"] == "decode":
        ctx, D, Hq = _spread(case, "ctx"), case["dim"], case["heads"] * case["group"]
        pages = sum(_blocks(c, B) for c in ctx)
        return {"bytes": sum(ctx) * 2 * H * D + pages * (2 * H * 4 + 4) + case["n"] * Hq * (D * 4 + 4)
                + (pages * H * 8 if case["mass"] else 0), "flops": 4 * D * Hq * sum(ctx)}
    ctx = _spread(case, "ctx")
    pages = [_blocks(c, B) for c in ctx]
    # every table and mass is read and written; evicted blocks are named
    return {"bytes": sum(pages) * (H * 8 + 12), "flops": sum(pages) * H}


# ---------------------------------------------------------------- inputs
def _pool(case, pages, gen, dev):
    """A cache in use: codes of normal values, scales that differ from block to block and head to head."""
    dtype, most = FORMATS[case["fmt"]]
    shape = (pages, 2, case["heads"], case["block"], case["dim"])
    codes = torch.empty(shape, dtype=dtype, device=dev)
    step = max(1, (1 << 27) // max(1, codes[0].numel()))
    for p in range(0, pages, step):
        x = torch.randn((min(step, pages - p),) + shape[1:], generator=gen, device=dev, dtype=torch.float32)
        x = (x * (most / 4)).clamp_(-most, most)
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


def _device_ints(values, dev, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device=dev)


def _offsets(lens, dev):
    return _device_ints(np.concatenate([[0], np.cumsum(lens)]).tolist(), dev, torch.int64)


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    n, H, B = case["n"], case["heads"], case["block"]
    state = {"case": case}

    def normal(*shape, spread=1.0):
        x = torch.randn(shape, generator=gen, device=dev, dtype=torch.float32) * spread
        return x.to(TYPES[case["dtype"]])

    if case["op"] == "append":
        new, ctx = _spread(case, "new"), _spread(case, "ctx")
        state["table"], pages = _tables(case, [c + t for c, t in zip(ctx, new)], 3, gen, dev, first=ctx)
        state["pages"], state["scales"] = _pool(case, pages, gen, dev)
        state["k"] = normal(sum(new), H, case["dim"], spread=2.0)
        state["v"] = normal(sum(new), H, case["dim"])
        state["offsets"], state["context"] = _offsets(new, dev), _device_ints(ctx, dev)
    elif case["op"] == "prefill":
        new, hit, Hq = _spread(case, "new"), _spread(case, "hit"), H * case["group"]
        state["new"], state["hit"] = new, hit
        if max(hit) > 0:
            state["table"], pages = _tables(case, hit, 3, gen, dev)
            state["pages"], state["scales"] = _pool(case, pages, gen, dev)
            state["prefix"] = _device_ints(hit, dev)
        state["q"] = normal(sum(new), Hq, case["dim"], spread=1.5)
        state["k"] = normal(sum(new), H, case["dim"])
        state["v"] = normal(sum(new), H, case["dim"])
        state["offsets"] = _offsets(new, dev)
        state["out"] = torch.empty_like(state["q"])
        state["lse"] = torch.empty(sum(new), Hq, dtype=torch.float32, device=dev)
    elif case["op"] == "decode":
        ctx, Hq = _spread(case, "ctx"), H * case["group"]
        state["ctx"] = ctx
        state["table"], pages = _tables(case, ctx, 3, gen, dev)
        state["pages"], state["scales"] = _pool(case, pages, gen, dev)
        state["q"] = normal(n, Hq, case["dim"], spread=1.5)
        state["context"] = _device_ints(ctx, dev)
        state["out"] = torch.empty_like(state["q"])
        state["lse"] = torch.empty(n, Hq, dtype=torch.float32, device=dev)
        if case["mass"]:     # what the steps before this one left
            width = state["table"].shape[1]
            state["mass_in"] = torch.rand(n, H, width, generator=gen, device=dev) * case["group"]
            live = torch.arange(width, device=dev)[None] * B < state["context"][:, None]
            state["mass_in"] *= live[:, None]
            state["mass"] = torch.empty_like(state["mass_in"])
    else:
        ctx = _spread(case, "ctx")
        blocks = [_blocks(c, B) for c in ctx]
        state["table"], _ = _tables(case, ctx, 3, gen, dev)
        width = state["table"].shape[1]
        # few blocks hold most of the weight; blocks that no token has looked at hold none
        mass = torch.rand(n, H, width, generator=gen, device=dev)
        mass = torch.where(mass < 0.2, torch.zeros_like(mass), mass ** 8 * 50)
        live = torch.arange(width, device=dev)[None] < _device_ints(blocks, dev)[:, None]
        state["table"] = torch.where(live, state["table"], torch.full_like(state["table"], -1))
        state["mass_in"] = (mass * live[:, None]).contiguous()
        state["context"] = _device_ints(ctx, dev)
        state["keep"] = _device_ints([max(1, int(b * case["keep"])) for b in blocks], dev)
        state["context_out"] = torch.empty_like(state["context"])
        state["table_out"] = torch.empty_like(state["table"])
        state["mass"] = torch.empty_like(state["mass_in"])
        state["freed"] = torch.empty_like(state["table"])
        state["num_freed"] = torch.empty_like(state["context"])
    if own:
        import paper_2607_02525_amd as P
        if "pages" in state:
            state["pool"] = P.KVPool(state["pages"], state["scales"])
        size = 0
        if case["op"] == "prefill":
            width = state["table"].shape[1] if "table" in state else 0
            size = P.peek_prefill_attention_workspace(n, sum(new), Hq, H, case["dim"], width * B)
        elif case["op"] == "decode":
            size = P.peek_decode_attention_workspace(state["pool"], n, Hq, state["table"].shape[1], mass=case["mass"])
        elif case["op"] == "evict":
            size = P.peek_kv_evict_workspace(n, H, state["table"].shape[1])
        state["workspace"] = torch.empty(max(size, 256), dtype=torch.uint8, device=dev)
    return state


def run(state):
    return (_run_own if own else _run_plain)[state["case"]["op"]](state)


# ---------------------------------------------------------------- the framework's operators
def _values(codes, scales):
    scales = scales[..., None, None]
    return codes * scales if codes.dtype == torch.int8 else codes.to(torch.float32).mul_(scales)


def _own_append(s):
    import paper_2607_02525_amd as P
    P.peek_kv_append(s["pool"], s["k"], s["v"], s["offsets"], s["context"], s["table"])
    return {"values": _values(s["pages"], s["scales"]), "scales": s["scales"]}


def _own_prefill(s):
    import paper_2607_02525_amd as P
    P.peek_prefill_attention(s["q"], s["k"], s["v"], s["offsets"], s["out"], s["workspace"], pool=s.get("pool"),
                             prefix=s.get("prefix"), block_table=s.get("table"), lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_decode(s):
    import paper_2607_02525_amd as P
    P.peek_decode_attention(s["pool"], s["q"], s["context"], s["table"], s["out"], s["workspace"], lse=s["lse"],
                            mass_in=s.get("mass_in"), mass=s.get("mass"))
    out = {"out": s["out"], "lse": s["lse"]}
    if "mass" in s:
        out["mass"] = s["mass"]
    return out


def _own_evict(s):
    import paper_2607_02525_amd as P
    c = s["case"]
    P.peek_kv_evict(s["context"], s["table"], s["mass_in"], s["keep"], c["block"], c["sink"], c["recent"],
                    s["context_out"], s["table_out"], s["mass"], s["freed"], s["num_freed"], s["workspace"])
    return {"context": s["context_out"], "table": s["table_out"], "mass": s["mass"], "freed": s["freed"],
            "num_freed": s["num_freed"]}


_run_own = {"append": _own_append, "prefill": _own_prefill, "decode": _own_decode, "evict": _own_evict}


# ---------------------------------------------------------------- plain forms, 32 bits
def _scale_of(amax, fmt):
    """fp8: the smallest power of two under which amax is no larger than 448. int8: amax / 127."""
    if fmt == "int8":
        return (amax / 127.0).clamp(SCALE_MIN, SCALE_MAX)
    m, e = torch.frexp(amax)
    e = torch.where(m <= 0.875, e - 9, e - 8)
    e = torch.where(amax > 0, e, torch.full_like(e, -60)).clamp(-60, 60)
    return torch.ldexp(torch.ones_like(amax), e)


def _codes_of(x, scale, fmt):
    dtype, most = FORMATS[fmt]
    x = (x / scale).clamp(-most, most)
    return (x.round() if fmt == "int8" else x).to(dtype)


def _plain_append(s):
    c, B = s["case"], s["case"]["block"]
    codes, scales, offsets, ctx = s["pages"], s["scales"], s["offsets"], s["context"]
    dev, P, total = codes.device, codes.shape[0], s["k"].shape[0]
    x = torch.stack([s["k"], s["v"]], 1).float()                          # [total, 2, H, D]
    row = torch.searchsorted(offsets, torch.arange(total, device=dev), right=True) - 1
    pos = ctx[row].long() + torch.arange(total, device=dev) - offsets[row]
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
    return {"values": _values(codes, scales), "scales": scales}


def _gathered(s, row, blocks):
    """K and V [H, blocks * B, D] of the leading blocks of a sequence."""
    ids = s["table"][row, :blocks].long()
    codes = s["pages"].view(torch.uint8)[ids].view(s["pages"].dtype)
    x = codes.float() * s["scales"][ids][..., None, None]                # [blocks, 2, H, B, D]
    x = x.permute(1, 2, 0, 3, 4).reshape(2, x.shape[2], -1, x.shape[4])
    return x[0], x[1]


def _plain_prefill(s):
    c = s["case"]
    G, H, D, B = c["group"], c["heads"], c["dim"], c["block"]
    q, k, v = s["q"], s["k"], s["v"]
    out, lse = torch.empty_like(q), torch.empty_like(s["lse"])
    at = 0
    for r, (t, h) in enumerate(zip(s["new"], s["hit"])):
        keys, values = (x[at:at + t].float().transpose(0, 1) for x in (k, v))
        if h:
            pk, pv = _gathered(s, r, h // B)
            keys, values = torch.cat([pk, keys], 1), torch.cat([pv, values], 1)
        keys = keys.transpose(1, 2).contiguous()
        step = max(1, (1 << 28) // (G * H * (t + h)))
        for i in range(0, t, step):
            m = min(step, t - i)
            x = q[at + i:at + i + m].float().view(m, H, G, D).permute(1, 2, 0, 3).reshape(H, G * m, D)
            logits = torch.matmul(x, keys[:, :, :h + i + m]) * (D ** -0.5)
            last = h + i + torch.arange(m, device=q.device).repeat(G)
            logits.masked_fill_(torch.arange(h + i + m, device=q.device)[None] > last[:, None], -math.inf)
            top = logits.amax(-1, keepdim=True)
            p = torch.exp(logits - top)
            total = p.sum(-1, keepdim=True)
            o = torch.matmul(p, values[:, :h + i + m].contiguous()) / total
            out[at + i:at + i + m] = o.view(H, G, m, D).permute(2, 0, 1, 3).reshape(m, H * G, D).to(q.dtype)
            lse[at + i:at + i + m] = (top + total.log()).view(H, G, m).permute(2, 0, 1).reshape(m, H * G)
        at += t
    return {"out": out, "lse": lse}


def _plain_decode(s):
    c = s["case"]
    n, G, H, D, B = c["n"], c["group"], c["heads"], c["dim"], c["block"]
    q, ctx = s["q"], s["context"]
    out, lse = torch.empty_like(q), torch.empty_like(s["lse"])
    mass = s["mass_in"].clone() if c["mass"] else None
    order = sorted(range(n), key=lambda r: s["ctx"][r])                  # sequences of like lengths together
    at = 0
    while at < n:
        some = [order[at]]
        while at + len(some) < n:
            longest = max(1, _blocks(s["ctx"][order[at + len(some)]], B))
            if (len(some) + 1) * longest * 2 * H * B * D > (1 << 29):
                break
            some.append(order[at + len(some)])
        at += len(some)
        width = max(1, _blocks(s["ctx"][some[-1]], B))
        rows = torch.tensor(some, device=q.device)
        ids = s["table"][rows, :width].long()
        codes = s["pages"].view(torch.uint8)[ids].view(s["pages"].dtype)
        x = codes.float() * s["scales"][ids][..., None, None]            # [rows, width, 2, H, B, D]
        x = x.permute(2, 0, 3, 1, 4, 5).reshape(2, len(some), H, width * B, D)
        keys, values = x[0], x[1]
        logits = torch.matmul(q[rows].float().view(len(some), H, G, D), keys.transpose(2, 3).contiguous()) * (D ** -0.5)
        dead = torch.arange(width * B, device=q.device)[None] >= ctx[rows][:, None]
        logits.masked_fill_(dead[:, None, None], -math.inf)
        top = logits.amax(-1, keepdim=True)
        p = torch.exp(logits - torch.where(top > -math.inf, top, torch.zeros_like(top)))
        total = p.sum(-1, keepdim=True)
        p = p / torch.where(total > 0, total, torch.ones_like(total))
        out[rows] = torch.matmul(p, values).reshape(len(some), H * G, D).to(q.dtype)
        lse[rows] = (top + total.log()).reshape(len(some), H * G)
        if mass is not None:
            mass[rows, :, :width] += p.sum(2).view(len(some), H, width, B).sum(-1)
    res = {"out": out, "lse": lse}
    if mass is not None:
        res["mass"] = mass
    return res


def _plain_evict(s):
    c = s["case"]
    n, H, B = c["n"], c["heads"], c["block"]
    table, mass, ctx = s["table"], s["mass_in"], s["context"]
    width, dev = table.shape[1], table.device
    blocks = (ctx + B - 1) // B
    score = mass[:, 0]
    for h in range(1, H):                                                # the sum's order is part of the definition
        score = score + mass[:, h]
    at = torch.arange(width, device=dev)[None]
    candidate = (at >= c["sink"]) & (at < (blocks - c["recent"])[:, None])
    drop = torch.minimum((blocks - s["keep"]).clamp(min=0), candidate.sum(1))
    order = torch.argsort(torch.where(candidate, score, torch.full_like(score, math.inf)), dim=1, stable=True)
    rank = torch.empty_like(order).scatter_(1, order, at.expand(n, -1))
    gone = candidate & (rank < drop[:, None])
    front = torch.argsort(gone.to(torch.int32), dim=1, stable=True)      # kept blocks first, in order
    kept = at < (width - drop)[:, None]
    table_out = torch.where(kept, table.gather(1, front), torch.full_like(table, -1))
    mass_out = torch.where(kept[:, None], mass.gather(2, front[:, None].expand(-1, H, -1)), torch.zeros_like(mass))
    back = torch.argsort((~gone).to(torch.int32), dim=1, stable=True)    # evicted blocks first, in order
    freed = torch.where(at < drop[:, None], table.gather(1, back), torch.full_like(table, -1))
    drop = drop.to(torch.int32)
    return {"context": ctx - drop * B, "table": table_out, "mass": mass_out, "freed": freed, "num_freed": drop}


_run_plain = {"append": _plain_append, "prefill": _plain_prefill, "decode": _plain_decode, "evict": _plain_evict}


# ---------------------------------------------------------------- from the definitions, in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "prefill": _exact_attention, "decode": _exact_attention,
            "evict": _exact_evict}[case["op"]](s)


def _rounded(x, scale, fmt):
    """x / scale as the format holds it: whole numbers to 127, or three bits after the leading one to 448."""
    y = x / scale
    if fmt == "int8":
        return y.clamp(-127, 127).round()
    exponent = (torch.frexp(y)[1].double() - 1).clamp(min=-6)
    unit = torch.exp2(exponent - 3)
    return ((y / unit).round() * unit).clamp(-448, 448)


def _exact_append(s):
    c = s["case"]
    B, fmt = c["block"], c["fmt"]
    held, scales = s["pages"].double(), s["scales"].double()
    table, starts, ctx = s["table"].tolist(), s["offsets"].tolist(), s["context"].tolist()
    both = torch.stack([s["k"], s["v"]], 1).double()
    most = FORMATS[fmt][1]
    if sum(starts[-1:]) // B + 2 * c["n"] > 20000:
        return None
    for r in range(c["n"]):
        first, last = ctx[r], ctx[r] + starts[r + 1] - starts[r]
        for b in range(first // B, _blocks(last, B)):
            lo, hi = max(first, b * B), min(last, (b + 1) * B)
            x = both[starts[r] + lo - first:starts[r] + hi - first].permute(1, 2, 0, 3)     # [2, H, tokens, D]
            p, at = table[r][b], lo - b * B
            top = x.abs().amax((2, 3))
            if fmt == "int8":
                new = top / most
            else:
                new = torch.exp2(torch.ceil(torch.log2((top / most).clamp(min=SCALE_MIN))))
            new = new.clamp(SCALE_MIN, SCALE_MAX)
            if at > 0:
                new = torch.maximum(new, scales[p])
                grown = (new > scales[p])[..., None, None]
                old = held[p, :, :, :at]
                again = _rounded(old * scales[p][..., None, None], new[..., None, None], fmt)
                held[p, :, :, :at] = torch.where(grown, again, old)
            scales[p] = new
            held[p, :, :, at:at + hi - lo] = _rounded(x, new[..., None, None], fmt)
    return {"values": held * scales[..., None, None], "scales": scales}


def _exact_attention(s):
    c = s["case"]
    G, H, D, B = c["group"], c["heads"], c["dim"], c["block"]
    if work(c)["flops"] > 2e13 or work(c)["bytes"] > 2e10:
        return None
    decode = c["op"] == "decode"
    new = [1] * c["n"] if decode else s["new"]
    held = s["ctx"] if decode else s["hit"]
    q = s["q"]
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device)
    mass = s["mass_in"].double() if c.get("mass") else None
    at = 0
    for r, (t, h) in enumerate(zip(new, held)):
        parts_k, parts_v = [], []
        if h:
            ids = s["table"][r, :_blocks(h, B)].tolist()
            where = torch.tensor(ids, device=q.device)
            codes = s["pages"].view(torch.uint8).index_select(0, where).view(s["pages"].dtype).double()
            x = codes * s["scales"].double().index_select(0, where)[..., None, None]
            parts_k.append(x[:, 0].transpose(1, 2).reshape(-1, H, D)[:h])
            parts_v.append(x[:, 1].transpose(1, 2).reshape(-1, H, D)[:h])
        if not decode:
            parts_k.append(s["k"][at:at + t].double())
            parts_v.append(s["v"][at:at + t].double())
        if not parts_k:
            at += t
            continue
        keys, values = torch.cat(parts_k), torch.cat(parts_v)
        seen = keys.shape[0]
        for head in range(H * G):
            kh, vh = keys[:, head // G].t().contiguous(), values[:, head // G].contiguous()
            step = max(1, (1 << 27) // seen)
            for i in range(0, t, step):
                rows = slice(at + i, at + min(i + step, t))
                x = q[rows, head].double() @ kh / math.sqrt(D)
                if not decode:
                    own_at = torch.arange(i, min(i + step, t), device=q.device)[:, None] + h
                    x = torch.where(torch.arange(seen, device=q.device)[None] <= own_at, x, -math.inf)
                lse[rows, head] = torch.logsumexp(x, 1)
                p = torch.exp(x - lse[rows, head][:, None])
                out[rows, head] = p @ vh
                if mass is not None:
                    whole = torch.zeros(_blocks(seen, B) * B, dtype=torch.float64, device=q.device)
                    whole[:seen] = p[0]
                    mass[r, head // G, :_blocks(seen, B)] += whole.view(-1, B).sum(1)
        at += t
    res = {"out": out, "lse": lse}
    if mass is not None:
        res["mass"] = mass
    return res


def _exact_evict(s):
    c = s["case"]
    B, sink, recent = c["block"], c["sink"], c["recent"]
    table, ctx, keep = (s[k].cpu().numpy() for k in ("table", "context", "keep"))
    mass = s["mass_in"].cpu().numpy()
    table_out, mass_out = np.full_like(table, -1), np.zeros(mass.shape)
    freed, ctx_out, count = np.full_like(table, -1), ctx.copy(), np.zeros_like(ctx)
    for r in range(c["n"]):
        blocks = _blocks(int(ctx[r]), B)
        score = np.zeros(table.shape[1], np.float32)
        for h in range(c["heads"]):          # 32 bits, heads in order: the operator's definition
            score = score + mass[r, h]
        able = list(range(sink, max(sink, blocks - recent)))
        able.sort(key=lambda b: (score[b], b))
        gone = sorted(able[:max(0, blocks - int(keep[r]))])
        stay = np.setdiff1d(np.arange(table.shape[1]), gone)
        table_out[r, :len(stay)] = table[r, stay]
        mass_out[r, :, :len(stay)] = mass[r][:, stay]
        freed[r, :len(gone)] = table[r, gone]
        count[r] = len(gone)
        ctx_out[r] -= B * len(gone)
    return {"context": torch.from_numpy(ctx_out), "table": torch.from_numpy(table_out),
            "mass": torch.from_numpy(mass_out), "freed": torch.from_numpy(freed), "num_freed": torch.from_numpy(count)}
