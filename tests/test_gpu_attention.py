"""GPU tests of the calls on the cache's contents (peek_kv_append,
peek_prefill_attention, peek_decode_attention, peek_kv_evict) against their
definitions in 64 bits (tests/kv_reference.py). Pages that no sequence names,
slots past a sequence's end and rows of no sequence hold NaN (or the format's
most negative code) throughout."""
import math

import numpy as np
import pytest

from tests import kv_reference as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
BF, HF, F8, I8 = torch.bfloat16, torch.float16, torch.float8_e4m3fn, torch.int8
JUNK = {F8: 0x7F, I8: 0x80}


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def make_pool(gen, tokens, H, B, D, fmt, spare=2, spread=2):
    """Codes and scales on the CPU, and the table that spreads sequences of these many tokens over shuffled pages."""
    blocks = [-(-t // B) for t in tokens]
    P, width = sum(blocks) + spare, max([1] + blocks)
    codes = torch.full((P, 2, H, B, D), JUNK[fmt], dtype=torch.uint8)
    scales = torch.full((P, 2, H), math.nan)
    ids = torch.randperm(P, generator=gen).tolist()
    table = torch.full((len(tokens), width), 0, dtype=torch.int32)
    at = 0
    for r, t in enumerate(tokens):
        for b in range(blocks[r]):
            p = ids[at]
            at += 1
            table[r, b] = p
            live = min(B, t - b * B)
            x = torch.randn(2, H, live, D, generator=gen)
            x = (x * 100).clamp(-448, 448).to(F8).view(torch.uint8) if fmt == F8 else \
                (x * 40).round().clamp(-127, 127).to(I8).view(torch.uint8)
            codes[p, :, :, :live] = x
            scales[p] = torch.exp2(torch.randint(-spread, spread + 1, (2, H), generator=gen).float()) / \
                (100 if fmt == F8 else 37)
    return codes.view(fmt), scales, table


def rows_of(gen, shape, dtype, layout, spread=1.0):
    """Values on the CPU, and the same on the GPU as a plain tensor or as a slice of a wider one."""
    x = (torch.randn(shape, generator=gen) * spread).to(dtype)
    if layout == "plain":
        return x, x.cuda()
    T, H, D = shape
    if layout == "fused":          # heads of q, k and v of a token side by side
        wide = torch.full((T, H + 3, D), math.nan, dtype=dtype).cuda()
        wide[:, 2:2 + H] = x.cuda()
        return x, wide[:, 2:2 + H]
    wide = torch.full((H, T, D + 8), math.nan, dtype=dtype).cuda()    # heads outermost, padded rows
    wide[:, :, :D] = x.cuda().transpose(0, 1)
    return x, wide[:, :, :D].transpose(0, 1)


def near(got, want, bound, what):
    got = got.double().cpu()
    assert got.shape == want.shape, what
    same = (got == want) | (got.isnan() & want.isnan())
    off = torch.where(same, torch.zeros_like(got), (got - want).abs())
    bad = ~(same | (off <= bound))
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {off.max().item():.3g}, " \
                          f"first at {bad.nonzero()[0].tolist()}"


# ------------------------------------------------------------------ decode
DECODE = [
    # contexts, kv heads, group, block, dim, dtype, format
    ([0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100], 2, 4, 16, 128, BF, F8),
    ([0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100], 2, 4, 16, 64, HF, I8),
    ([3, 4, 5, 0, 129, 255, 256, 257, 1000], 1, 1, 4, 128, HF, F8),
    ([7, 8, 9, 500], 3, 5, 8, 64, BF, I8),
    ([300, 31, 0, 2049], 1, 8, 32, 128, BF, I8),
    ([128, 127, 129, 640], 2, 16, 64, 128, HF, I8),
    ([5, 1023], 2, 17, 128, 64, BF, F8),
    ([256, 255, 257, 1], 1, 40, 256, 128, BF, F8),
    ([4500], 2, 3, 16, 128, BF, F8),
    ([9001], 1, 7, 16, 64, HF, F8),
    ([20000, 0, 11], 1, 4, 256, 128, BF, I8),
    ([0, 0, 0], 2, 2, 16, 128, BF, F8),
]


def run_decode(gen, contexts, H, G, B, D, dtype, fmt, layout="plain", with_mass=True, scale=None, extra_columns=0,
               spread=2, q_spread=1.0, stream=None):
    import paper_2607_02525_amd as P
    n, Hq = len(contexts), H * G
    codes, scales, table = make_pool(gen, contexts, H, B, D, fmt, spread=spread)
    q, dq = rows_of(gen, (n, Hq, D), dtype, layout, q_spread)
    pool = P.KVPool(codes.cuda(), scales.cuda())
    W = table.shape[1]
    # the table is the leading columns of a wider one
    wide = torch.full((n, W + extra_columns), 0, dtype=torch.int32)
    wide[:, :W] = table
    dtable = wide.cuda()[:, :W]
    _, out = rows_of(gen, (n, Hq, D), dtype, layout)
    lse = torch.full((n, Hq), math.nan).cuda()
    mass_in = torch.rand(n, H, W, generator=gen) if with_mass else None
    mass = torch.full((n, H, W), math.nan).cuda() if with_mass else None
    ctx = torch.tensor(contexts, dtype=torch.int32).cuda()
    ws = torch.full((max(256, P.peek_decode_attention_workspace(pool, n, Hq, W, mass=with_mass)),), 0xFF,
                    dtype=torch.uint8).cuda()
    args = (pool, dq, ctx, dtable, out, ws)
    kw = dict(scale=scale, lse=lse, mass_in=mass_in.cuda() if with_mass else None, mass=mass)
    torch.cuda.synchronize()
    P.peek_decode_attention(*args, stream=stream, **kw)
    torch.cuda.synchronize()
    s, most = D ** -0.5 if scale is None else scale, R.most_of(scales, fmt)
    for r, c in enumerate(contexts):
        k, v = R.cached(codes, scales, table[r], c)
        want, wl, w, spread_, reach = R.attend(q[r:r + 1], k, v, s, c)
        near(out[r:r + 1], want, R.out_bound(want, spread_, reach, dtype, c, most), f"out of sequence {r} ({c} tokens)")
        near(lse[r:r + 1], wl, R.lse_bound(wl, reach, D), f"lse of sequence {r} ({c} tokens)")
        if with_mass:
            nb = -(-c // B)
            add = torch.zeros(H, W, dtype=torch.float64)
            whole = torch.zeros(Hq, max(nb, 1) * B, dtype=torch.float64)
            whole[:, :c] = w[:, 0]
            add[:, :nb] = whole.view(H, G, max(nb, 1), B).sum((1, 3))[:, :nb]
            total = mass_in[r].double() + add
            near(mass[r], total, R.mass_bound(add, reach.view(H, G).amax(1)[:, None], total), f"mass of sequence {r}")
    return args, kw


@pytest.mark.parametrize("case", range(len(DECODE)))
def test_decode(case):
    contexts, *rest = DECODE[case]
    print("[gpu] decode", DECODE[case], flush=True)
    run_decode(torch.Generator().manual_seed(case), contexts, *rest)


@pytest.mark.parametrize("layout", ["fused", "outer"])
@pytest.mark.parametrize("with_mass", [False, True])
def test_decode_layouts(layout, with_mass):
    run_decode(torch.Generator().manual_seed(7), [40, 0, 333], 2, 5, 16, 128, BF, F8, layout=layout,
               with_mass=with_mass, extra_columns=5)


@pytest.mark.parametrize("fmt", [F8, I8])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_decode_extreme_scales_and_sharp_rows(fmt, dtype):
    """Scales 2^24 apart inside a sequence, and logits so far apart that one token takes all the weight."""
    gen = torch.Generator().manual_seed(3)
    run_decode(gen, [700, 65], 2, 4, 16, 128, dtype, fmt, spread=12 if dtype == BF else 6, scale=1e-4)
    run_decode(gen, [700, 65], 2, 4, 16, 128, dtype, fmt, q_spread=40.0)
    run_decode(gen, [700, 65], 2, 4, 16, 128, dtype, fmt, scale=0.0)
    run_decode(gen, [700, 65], 2, 4, 16, 128, dtype, fmt, scale=-0.05)


def test_decode_is_deterministic_and_mass_may_be_in_place():
    import paper_2607_02525_amd as P
    args, kw = run_decode(torch.Generator().manual_seed(5), [3000, 77, 512], 2, 8, 16, 128, BF, F8)
    first = [args[4].clone(), kw["lse"].clone(), kw["mass"].clone()]
    for _ in range(3):
        P.peek_decode_attention(*args, **kw)
        assert all(torch.equal(a, b) for a, b in zip(first, (args[4], kw["lse"], kw["mass"])))
    kw["mass"] = kw["mass_in"]
    P.peek_decode_attention(*args, **kw)
    assert torch.equal(kw["mass"], first[2])


def test_decode_on_another_stream():
    s = torch.cuda.Stream()
    run_decode(torch.Generator().manual_seed(6), [900, 77], 2, 4, 16, 128, BF, F8, stream=s)


def test_pages_past_32_bit_offsets():
    """A pool of more than 4 GiB: its last pages are written, read back and attended to."""
    import paper_2607_02525_amd as P
    H, B, D, N = 8, 16, 128, 33 * (1 << 12)
    assert N * 2 * H * B * D > 1 << 32
    pool = P.KVPool.empty(N, H, B, D)
    gen = torch.Generator().manual_seed(1)
    T = 40
    k, dk = rows_of(gen, (T, H, D), BF, "plain")
    v, dv = rows_of(gen, (T, H, D), BF, "plain")
    table = torch.tensor([[N - 1, 5, N - 2]], dtype=torch.int32)
    zero = torch.zeros(1, dtype=torch.int32).cuda()
    P.peek_kv_append(pool, dk, dv, torch.tensor([0, T]).cuda(), zero, table.cuda())
    ids = table[0].long().cuda()
    pages = pool.pages.view(torch.uint8)[ids].view(F8).cpu()
    scales = pool.scales[ids].cpu()
    gk, gv = R.cached(pages, scales, [0, 1, 2], T)
    assert (gk - k.double()).abs().max() < 0.3 and (gv - v.double()).abs().max() < 0.3
    q, dq = rows_of(gen, (1, 2 * H, D), BF, "plain")
    out = torch.empty_like(dq)
    ws = torch.empty(max(256, P.peek_decode_attention_workspace(pool, 1, 2 * H, 3)), dtype=torch.uint8).cuda()
    P.peek_decode_attention(pool, dq, torch.tensor([T], dtype=torch.int32).cuda(), table.cuda(), out, ws)
    want, _, _, spread, reach = R.attend(q, gk, gv, D ** -0.5, T)
    near(out, want, R.out_bound(want, spread, reach, BF), "out")


# ----------------------------------------------------------------- prefill
PREFILL = [
    # (prefix, new) of every sequence, kv heads, group, block, dim, dtype, format
    ([(0, 1), (0, 2), (0, 0), (0, 31), (0, 32), (0, 33), (0, 64), (0, 65)], 2, 4, 16, 128, BF, F8),
    ([(0, 127), (0, 128), (0, 129), (0, 1)], 1, 1, 16, 128, HF, F8),
    ([(0, 300), (0, 0), (0, 77)], 2, 3, 16, 64, BF, I8),
    ([(16, 1), (32, 0), (0, 5), (512, 64), (48, 130)], 2, 4, 16, 128, BF, F8),
    ([(512, 3), (16, 200), (1008, 40)], 1, 5, 16, 128, HF, I8),
    ([(4, 1), (12, 30), (256, 17)], 3, 2, 4, 64, HF, F8),
    ([(5, 9), (63, 3), (65, 70), (1, 1)], 1, 8, 8, 128, BF, I8),        # prefixes that end inside a block
    ([(256, 33), (300, 100)], 2, 1, 256, 64, BF, F8),
    ([(2048, 5)], 1, 16, 32, 128, BF, F8),
    ([(6000, 2)], 1, 8, 64, 64, HF, I8),
    ([(0, 700)], 1, 7, 16, 128, BF, F8),
    ([(100, 1), (3, 1), (0, 1)], 1, 33, 16, 128, BF, F8),
    ([(0, 0), (16, 0)], 1, 4, 16, 128, BF, F8),
    ([(0, 2100)], 1, 1, 16, 64, BF, F8),       # few tiles: keys in parts, of which early rows see one
    ([(1500, 600), (0, 40)], 1, 2, 16, 128, HF, F8),
    ([(0, 0), (6000, 3), (0, 0), (500, 9), (0, 1), (2300, 260), (0, 0)], 2, 2, 16, 128, BF, I8),
    ([(48 * i, i % 3) for i in range(64)], 1, 4, 16, 64, BF, F8),
]


def run_prefill(gen, seqs, H, G, B, D, dtype, fmt, layout="plain", scale=None, cache=True, slack=3, q_spread=1.0,
                spread=2):
    import paper_2607_02525_amd as P
    n, Hq = len(seqs), H * G
    held, new = [s[0] for s in seqs], [s[1] for s in seqs]
    codes, scales, table = make_pool(gen, held, H, B, D, fmt, spread=spread)
    T = sum(new) + slack                       # rows past the last sequence belong to nobody
    qkv = []
    for heads, s in ((Hq, q_spread), (H, 1.0), (H, 1.0)):
        x, dx = rows_of(gen, (T, heads, D), dtype, layout, s)
        if slack:
            dx[T - slack:] = math.nan
        qkv.append((x, dx))
    (q, dq), (k, dk), (v, dv) = qkv
    offsets = np.concatenate([[0], np.cumsum(new)])
    _, out = rows_of(gen, (T, Hq, D), dtype, layout)
    out.fill_(-7)
    lse = torch.full((T, Hq), -7.0).cuda()
    more, width = {}, 0
    if cache:
        width = table.shape[1]
        more = dict(pool=P.KVPool(codes.cuda(), scales.cuda()), prefix=torch.tensor(held, dtype=torch.int32).cuda(),
                    block_table=table.cuda())
    else:
        assert not any(held)
    ws = torch.full((max(256, P.peek_prefill_attention_workspace(n, T, Hq, H, D, width * B)),), 0xFF,
                    dtype=torch.uint8).cuda()
    doff = torch.tensor(offsets.tolist(), dtype=torch.int64).cuda()
    P.peek_prefill_attention(dq, dk, dv, doff, out, ws, scale=scale, lse=lse, **more)
    torch.cuda.synchronize()
    s, most = D ** -0.5 if scale is None else scale, R.most_of(scales, fmt)
    for r in range(n):
        a, b = int(offsets[r]), int(offsets[r + 1])
        pk, pv = R.cached(codes, scales, table[r], held[r])
        want, wl, _, spread_, reach = R.attend(q[a:b], torch.cat([pk, k[a:b].double()]),
                                               torch.cat([pv, v[a:b].double()]), s, held[r] + 1)
        near(out[a:b], want, R.out_bound(want, spread_, reach, dtype, held[r] + new[r], most),
             f"out of sequence {r} {seqs[r]}")
        near(lse[a:b], wl, R.lse_bound(wl, reach, D), f"lse of sequence {r} {seqs[r]}")
    assert (out[sum(new):] == -7).all() and (lse[sum(new):] == -7).all(), "rows of no sequence were written"
    return (dq, dk, dv, doff, out, ws), dict(scale=scale, lse=lse, **more)


@pytest.mark.parametrize("case", range(len(PREFILL)))
def test_prefill(case):
    seqs, *rest = PREFILL[case]
    print("[gpu] prefill", PREFILL[case], flush=True)
    run_prefill(torch.Generator().manual_seed(case), seqs, *rest, cache=any(s[0] for s in seqs))


@pytest.mark.parametrize("layout", ["fused", "outer"])
def test_prefill_layouts(layout):
    run_prefill(torch.Generator().manual_seed(2), [(32, 40), (0, 90), (16, 0), (160, 3)], 2, 4, 16, 128, BF, F8,
                layout=layout)


@pytest.mark.parametrize("dtype,fmt", [(BF, F8), (HF, I8)])
def test_prefill_sharp_flat_and_extreme(dtype, fmt):
    gen = torch.Generator().manual_seed(4)
    seqs = [(48, 70), (0, 40), (320, 9)]
    run_prefill(gen, seqs, 2, 4, 16, 128, dtype, fmt, q_spread=40.0)
    run_prefill(gen, seqs, 2, 4, 16, 128, dtype, fmt, scale=0.0)
    run_prefill(gen, seqs, 2, 4, 16, 128, dtype, fmt, scale=-0.05)
    run_prefill(gen, seqs, 2, 4, 16, 128, dtype, fmt, spread=12 if dtype == BF else 6, scale=1e-4)


def test_prefill_with_a_cache_in_which_nothing_was_found():
    run_prefill(torch.Generator().manual_seed(8), [(0, 50), (0, 3)], 2, 2, 16, 64, BF, F8, cache=True)


def test_prefill_is_deterministic_and_may_run_on_another_stream():
    import paper_2607_02525_amd as P
    args, kw = run_prefill(torch.Generator().manual_seed(9), [(480, 7), (0, 300), (64, 64)], 2, 4, 16, 128, BF, F8)
    first = args[4].clone(), kw["lse"].clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        P.peek_prefill_attention(*args, stream=s, **kw)
        s.synchronize()
        assert torch.equal(args[4], first[0]) and torch.equal(kw["lse"], first[1])


def test_decode_equals_a_prefill_of_one_token():
    """The last token of a prompt, once by each call over the same cache (its own K and V: codes both know exactly)."""
    import paper_2607_02525_amd as P
    gen = torch.Generator().manual_seed(10)
    H, G, B, D, ctx = 2, 4, 16, 128, 481
    codes, scales, table = make_pool(gen, [ctx], H, B, D, F8)
    pk, pv = R.cached(codes, scales, table[0], ctx)
    q, dq = rows_of(gen, (1, H * G, D), BF, "plain")
    pool = P.KVPool(codes.cuda(), scales.cuda())
    outs = []
    for out in (torch.empty_like(dq), torch.empty_like(dq)):
        if not outs:
            ws = torch.empty(P.peek_decode_attention_workspace(pool, 1, H * G, table.shape[1]) + 256,
                             dtype=torch.uint8).cuda()
            P.peek_decode_attention(pool, dq, torch.tensor([ctx], dtype=torch.int32).cuda(), table.cuda(), out, ws)
        else:
            ws = torch.empty(P.peek_prefill_attention_workspace(1, 1, H * G, H, D, table.shape[1] * B) + 256,
                             dtype=torch.uint8).cuda()
            P.peek_prefill_attention(dq, pk[-1:].to(BF).cuda(), pv[-1:].to(BF).cuda(), torch.tensor([0, 1]).cuda(), out,
                                     ws, pool=pool, prefix=torch.tensor([ctx - 1], dtype=torch.int32).cuda(),
                                     block_table=table.cuda())
        outs.append(out)
    want, _, _, spread, reach = R.attend(q, pk, pv, D ** -0.5, ctx)
    for out in outs:
        near(out, want, R.out_bound(want, spread, reach, BF), "out")


@pytest.mark.parametrize("dtype,D", [(BF, 128), (HF, 64)])
def test_prefill_does_not_see_later_tokens_whatever_they_hold(dtype, D):
    """NaN and infinities in K and V of some tokens: rows before them are as if they were not there; rows from
    them on have what the sums give (an infinity of one sign, or NaN), element by element."""
    import paper_2607_02525_amd as P
    gen = torch.Generator().manual_seed(15)
    H, G, new = 2, 4, [150, 70]
    T = sum(new)
    q, k, v = ((torch.randn(T, h, D, generator=gen)).to(dtype) for h in (H * G, H, H))
    v[20, 0, 3], v[21, 0, 4], v[40, 0, 4], v[100, 0, 5] = math.nan, math.inf, -math.inf, -math.inf
    v[63, 0, 7], v[149, 0], k[130, 0, 1], v[160, 1, 9] = math.inf, math.nan, math.nan, math.nan
    doff = torch.tensor([0, 150, 220]).cuda()
    dq = q.cuda()
    out, lse = torch.empty_like(dq), torch.empty(T, H * G).cuda()
    ws = torch.empty(P.peek_prefill_attention_workspace(2, T, H * G, H, D, 0) + 256, dtype=torch.uint8).cuda()
    P.peek_prefill_attention(dq, k.cuda(), v.cuda(), doff, out, ws, lse=lse)
    for a, b in ((0, 150), (150, 220)):
        for i in range(a, b):
            want, wl, _, spread, reach = R.attend(q[i:i + 1], k[a:i + 1], v[a:i + 1], D ** -0.5, i - a + 1)
            bound = R.out_bound(want, spread, reach, dtype, i - a + 1, 8.0).nan_to_num(0, 0)
            near(out[i:i + 1], want, bound, f"out of row {i - a}")
            near(lse[i:i + 1], wl, R.lse_bound(wl, reach, D).nan_to_num(0, 0), f"lse of row {i - a}")


def test_many_short_sequences():
    """More sequences than one look of 64 places, or two, can tell apart."""
    gen = torch.Generator().manual_seed(14)
    for n in (65, 4097, 6000):
        lens = torch.randint(0, 4, (n,), generator=gen).tolist()
        held = (torch.randint(0, 3, (n,), generator=gen) * 4).tolist()
        seqs = list(zip(held, lens))
        run_prefill(gen, seqs, 1, 1, 4, 64, BF, I8)
        run_append(gen, seqs, 1, 4, 64, BF, F8)
        run_decode(gen, held, 1, 2, 4, 64, HF, F8)


# ------------------------------------------------------------------ append
APPEND = [
    # (cached before, new), kv heads, block, dim, dtype, format
    ([(0, 1), (1, 1), (15, 1), (16, 1), (17, 15), (31, 2), (7, 0)], 2, 16, 128, BF, F8),
    ([(0, 1), (1, 1), (15, 1), (16, 1), (17, 15), (31, 2), (7, 0)], 3, 16, 64, HF, I8),
    ([(0, 100), (3, 9), (4, 4), (5, 1)], 1, 4, 128, HF, F8),
    ([(250, 10), (0, 600), (256, 1), (511, 2)], 2, 256, 64, BF, I8),
    ([(8, 200), (0, 0), (13, 50)], 5, 8, 128, BF, F8),
    ([(40, 90)], 1, 64, 128, HF, I8),
    ([(100, 33), (31, 33)], 2, 32, 64, BF, F8),
    ([(100, 300), (1, 130)], 2, 128, 128, BF, I8),
]


def run_append(gen, seqs, H, B, D, dtype, fmt, layout="plain", spread=1.0, poison=None):
    import paper_2607_02525_amd as P
    ctx, new = [s[0] for s in seqs], [s[1] for s in seqs]
    codes, scales, table = make_pool(gen, [a + b for a, b in seqs], H, B, D, fmt)
    offsets = [0] + np.cumsum(new).tolist()
    T = offsets[-1]
    # magnitudes that differ from token to token, so that scales grow and stay
    size = torch.exp2(torch.randint(-6, 7, (T, 1, 1), generator=gen).float()) * spread
    both = []
    for _ in range(2):
        x = (torch.randn(T, H, D, generator=gen) * size).to(dtype)
        if poison is not None:
            poison(x)
        _, dx = rows_of(gen, (T, H, D), dtype, layout)
        dx.copy_(x)
        both.append((x, dx))
    pool = P.KVPool(codes.cuda(), scales.cuda())
    P.peek_kv_append(pool, both[0][1], both[1][1], torch.tensor(offsets).cuda(),
                     torch.tensor(ctx, dtype=torch.int32).cuda(), table.cuda())
    torch.cuda.synchronize()
    want, ws = codes.double().numpy(), scales.double().numpy().copy()
    R.append(want, ws, both[0][0].double().numpy(), both[1][0].double().numpy(), offsets, ctx, table.tolist(), fmt)
    got_codes, got_scales = pool.pages.double().cpu().numpy(), pool.scales.double().cpu().numpy()
    np.testing.assert_array_equal(got_scales, ws)
    np.testing.assert_array_equal(got_codes, want)


@pytest.mark.parametrize("case", range(len(APPEND)))
def test_append(case):
    seqs, *rest = APPEND[case]
    print("[gpu] append", APPEND[case], flush=True)
    run_append(torch.Generator().manual_seed(case), seqs, *rest)


@pytest.mark.parametrize("layout", ["fused", "outer"])
@pytest.mark.parametrize("fmt", [F8, I8])
def test_append_layouts(layout, fmt):
    run_append(torch.Generator().manual_seed(11), [(5, 40), (0, 17)], 2, 16, 64, BF, fmt, layout=layout)


@pytest.mark.parametrize("fmt", [F8, I8])
def test_append_zeros_tiny_huge_and_nonfinite_values(fmt):
    gen = torch.Generator().manual_seed(12)
    seqs = [(3, 30), (0, 33)]
    run_append(gen, seqs, 2, 16, 64, BF, fmt, spread=0.0)
    run_append(gen, seqs, 2, 16, 64, BF, fmt, spread=2.0 ** -90)       # below the smallest scale
    run_append(gen, seqs, 2, 16, 64, BF, fmt, spread=2.0 ** 100)       # above the largest
    run_append(gen, seqs, 2, 16, 64, HF, fmt, spread=2.0 ** -20)       # subnormal inputs

    def poison(x):
        x[4, :, 3], x[5, 1, 7], x[20, 0], x[21, 0, 2] = math.inf, -math.inf, math.nan, math.inf
    run_append(gen, seqs, 2, 16, 64, BF, fmt, poison=poison)


def test_append_one_token_at_a_time_fills_a_block():
    """Sixteen appends of one token: the scale never falls, and older codes are those that the definition gives."""
    import paper_2607_02525_amd as P
    gen = torch.Generator().manual_seed(13)
    H, B, D = 2, 16, 128
    for fmt in (F8, I8):
        pool = P.KVPool(torch.zeros(1, 2, H, B, D, dtype=torch.uint8).view(fmt).cuda(), torch.ones(1, 2, H).cuda())
        want, ws = np.zeros((1, 2, H, B, D)), np.ones((1, 2, H))
        off, table = torch.tensor([0, 1]).cuda(), torch.zeros(1, 1, dtype=torch.int32).cuda()
        for t in range(B):
            k = (torch.randn(1, H, D, generator=gen) * 2.0 ** float(torch.randint(-3, 4, (1,), generator=gen))).to(BF)
            v = torch.randn(1, H, D, generator=gen).to(BF)
            P.peek_kv_append(pool, k.cuda(), v.cuda(), off, torch.tensor([t], dtype=torch.int32).cuda(), table)
            R.append(want, ws, k.double().numpy(), v.double().numpy(), [0, 1], [t], [[0]], fmt)
            np.testing.assert_array_equal(pool.scales.double().cpu().numpy(), ws)
            np.testing.assert_array_equal(pool.pages.double().cpu().numpy(), want)


def test_append_leaves_out_blocks_without_a_page():
    """Page ids outside the pool and tokens past the table: nothing is written for them, the rest is."""
    import paper_2607_02525_amd as P
    H, B, D = 1, 4, 64
    pool = P.KVPool(torch.full((3, 2, H, B, D), 9, dtype=torch.int8).cuda(), torch.full((3, 2, H), 5.0).cuda())
    k = torch.ones(16, H, D, dtype=BF).cuda()
    table = torch.tensor([[1, -1, 7]], dtype=torch.int32).cuda()
    P.peek_kv_append(pool, k, k, torch.tensor([0, 16]).cuda(), torch.zeros(1, dtype=torch.int32).cuda(), table)
    assert (pool.pages[1] == 127).all() and (pool.pages[[0, 2]] == 9).all()
    assert (pool.scales[[0, 2]] == 5).all() and (pool.scales[1] < 1).all()


# ---------------------------------------------------------------- eviction
EVICT = [
    # contexts, kv heads, block, keep, sink, recent
    ([0, 1, 16, 17, 100, 1000, 5000], 2, 16, [1, 1, 1, 1, 3, 20, 300], 1, 2),
    ([0, 1, 16, 17, 100, 1000, 5000], 1, 16, [0, 0, 0, 0, 0, 0, 0], 0, 1),
    ([5000, 4000, 4100], 8, 4, [600, 1000, 5], 3, 4),
    ([260, 70000], 3, 256, [1, 100], 0, 1),
    ([90000, 8, 33000], 4, 16, [2000, 1, 2063], 1, 4),
    ([300, 300], 2, 16, [4, 19], 100, 1),           # sinks protect everything
    ([300, 300], 2, 16, [4, -3], 0, 2000000000),    # so do recent blocks
]


def run_evict(contexts, H, B, keep, sink, recent, kind, seed=0, spare_columns=3):
    import paper_2607_02525_amd as P
    rng = np.random.default_rng(seed)
    n, W = len(contexts), max(1, max(-(-c // B) for c in contexts)) + spare_columns
    table = rng.permutation(n * W).astype(np.int32).reshape(n, W)
    mass = rng.random((n, H, W), dtype=np.float32)
    if kind == "ties":
        mass = np.floor(mass * 3).astype(np.float32)
    elif kind == "sparse":
        mass = np.where(mass < 0.6, 0, mass ** 9 * 1e4).astype(np.float32)
    elif kind == "odd":      # negative zero, infinities, NaN, negative and subnormal values
        mass = rng.choice(np.array([0.0, -0.0, np.inf, np.nan, -1.0, 1e-42, 3.5, 3.5], np.float32), mass.shape)
        mass[:, 1:] = np.where(np.isinf(mass[:, 1:]), 0, mass[:, 1:])
    wide = torch.full((n, W + 2), -9, dtype=torch.int32)
    wide[:, :W] = torch.from_numpy(table)
    ctx = torch.tensor(contexts, dtype=torch.int32).cuda()
    out = [torch.full((n, W), -5, dtype=torch.int32).cuda(), torch.full((n, H, W), -5.0).cuda(),
           torch.full((n, W), -5, dtype=torch.int32).cuda(), torch.full((n,), -5, dtype=torch.int32).cuda()]
    ws = torch.full((max(256, P.peek_kv_evict_workspace(n, H, W)),), 0xFF, dtype=torch.uint8).cuda()
    P.peek_kv_evict(ctx, wide.cuda()[:, :W], torch.from_numpy(mass).cuda(),
                    torch.tensor(keep, dtype=torch.int32).cuda(), B, sink, recent, ctx, *out, ws)  # context in place
    torch.cuda.synchronize()
    c, t, m, f, k = R.evict(contexts, table, mass, keep, B, sink, recent)
    np.testing.assert_array_equal(out[3].cpu().numpy(), k)
    np.testing.assert_array_equal(ctx.cpu().numpy(), c)
    np.testing.assert_array_equal(out[2].cpu().numpy(), f)
    np.testing.assert_array_equal(out[0].cpu().numpy(), t)
    np.testing.assert_array_equal(out[1].cpu().numpy(), m)


@pytest.mark.parametrize("kind", ["plain", "ties", "sparse", "odd"])
@pytest.mark.parametrize("case", range(len(EVICT)))
def test_evict(case, kind):
    print("[gpu] evict", EVICT[case], kind, flush=True)
    run_evict(*EVICT[case], kind, seed=case)


@pytest.mark.parametrize("kind", ["ties", "sparse", "odd"])
def test_evict_of_wide_tables(kind):
    run_evict([36000, 0, 33001, 8, 34500], 9, 4, [4000, 1, 8250, 1, 0], 3, 2, kind)


def test_evict_of_a_row_of_a_million_tokens():
    run_evict([1000000, 5], 2, 4, [70000, 1], 1, 4, "plain")


def test_evict_of_tables_without_columns():
    import paper_2607_02525_amd as P
    i32 = dict(dtype=torch.int32, device="cuda")
    empty = torch.empty(2, 0, **i32)
    mass = torch.empty(2, 1, 0, device="cuda")
    ctx, count = torch.zeros(2, **i32), torch.full((2,), -5, **i32)
    P.peek_kv_evict(ctx, empty, mass, torch.zeros(2, **i32), 16, 0, 1, ctx, torch.empty(2, 0, **i32),
                    torch.empty_like(mass), torch.empty(2, 0, **i32), count, None)
    torch.cuda.synchronize()
    assert count.tolist() == [0, 0] and ctx.tolist() == [0, 0]


# ---------------------------------------------------------- serving together
def test_serving_steps_in_a_graph():
    """Append, decode with weights and eviction captured once and replayed: every replay equals the eager calls."""
    import paper_2607_02525_amd as P
    gen = torch.Generator().manual_seed(20)
    H, G, B, D, n = 2, 4, 16, 128, 3
    contexts = [200, 37, 900]
    codes, scales, table = make_pool(gen, [c + 1 for c in contexts], H, B, D, F8)
    pages0, scales0 = codes.cuda(), scales.cuda()
    pool = P.KVPool(pages0.clone(), scales0.clone())
    k, v, q = (rows_of(gen, (n, h, D), BF, "plain")[1] for h in (H, H, H * G))
    dtable, W = table.cuda(), table.shape[1]
    before = torch.tensor(contexts, dtype=torch.int32).cuda()
    after, off = before + 1, torch.arange(n + 1).cuda()
    out, lse = torch.empty_like(q), torch.empty(n, H * G).cuda()
    mass_in, mass = torch.rand(n, H, W, generator=gen).cuda(), torch.empty(n, H, W).cuda()
    keep = torch.tensor([8, 8, 8], dtype=torch.int32).cuda()
    res = [torch.empty_like(before), torch.empty_like(dtable), torch.empty_like(mass), torch.empty_like(dtable),
           torch.empty_like(before)]
    ws = torch.empty(P.peek_decode_attention_workspace(pool, n, H * G, W, mass=True) + 256, dtype=torch.uint8).cuda()
    ws2 = torch.empty(P.peek_kv_evict_workspace(n, H, W) + 256, dtype=torch.uint8).cuda()

    def step():
        P.peek_kv_append(pool, k, v, off, before, dtable)
        P.peek_decode_attention(pool, q, after, dtable, out, ws, lse=lse, mass_in=mass_in, mass=mass)
        P.peek_kv_evict(after, dtable, mass, keep, B, 1, 2, *res, ws2)

    outputs = [pool.pages.view(torch.uint8), pool.scales, out, lse, mass, *res]
    step()
    torch.cuda.synchronize()
    want = [x.clone() for x in outputs]

    def reset():
        pool.pages.view(torch.uint8).copy_(pages0.view(torch.uint8))
        pool.scales.copy_(scales0)
        for x in outputs[2:]:
            x.fill_(3)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for rep in range(4):
        reset()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(outputs, want)):
            assert torch.equal(a.nan_to_num(5), b.nan_to_num(5)), f"replay {rep}: output {i}"
        step()
        torch.cuda.synchronize()


def test_validation_reports_broken_preconditions(monkeypatch):
    import paper_2607_02525_amd as P
    monkeypatch.setenv("PEEK_VALIDATE", "1")
    pool = P.KVPool(torch.zeros(4, 2, 1, 16, 64, dtype=torch.int8).cuda(), torch.ones(4, 2, 1).cuda())
    i32 = dict(dtype=torch.int32, device="cuda")
    q = torch.zeros(1, 2, 64, dtype=BF, device="cuda")
    k = torch.zeros(1, 1, 64, dtype=BF, device="cuda")
    out = torch.empty_like(q)
    ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    good = torch.tensor([[0, 3]], **i32)
    one = torch.tensor([0, 1], device="cuda")

    def status(call):
        with pytest.raises(P.PeekError) as e:
            call()
        return e.value.status, str(e.value)

    P.peek_decode_attention(pool, q, torch.tensor([32], **i32), good, out, ws)
    outside, none = torch.tensor([[0, 4]], **i32), torch.tensor([[-1, 0]], **i32)
    for ctx, table in ((33, good), (-1, good), (32, outside), (32, none)):
        held = torch.tensor([ctx], **i32)
        calls = [lambda: P.peek_decode_attention(pool, q, held, table, out, ws),
                 lambda: P.peek_prefill_attention(q, k, k, one, out, ws, pool=pool, prefix=held, block_table=table)]
        for call in calls:
            s, message = status(call)
            assert s == P.PEEK_ERR_INVALID_ARGUMENT and ("table" in message), message
    assert status(lambda: P.peek_kv_append(pool, k, k, one, torch.tensor([32], **i32), good))[0] == -1
    bad = torch.tensor([0, 2], device="cuda")
    assert "offsets" in status(lambda: P.peek_kv_append(pool, k, k, bad, torch.tensor([0], **i32), good))[1]
    assert "offsets" in status(lambda: P.peek_prefill_attention(q, k, k, bad, out, ws))[1]
