"""GPU tests of peek_shared_decode_attention against its definition in 64 bits (tests/kv_reference.py). Slots past a
sequence's end, pages that no sequence names and a member's own entries for what it shares lead to NaN."""
import math

import pytest

from tests import kv_reference as R
from tests.test_gpu_attention import BF, F8, HF, I8, JUNK, near, rows_of

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def grouped_pool(gen, groups, B, H, D, fmt, spread=2):
    """groups: (tokens shared, [own tokens of each member]) -> codes, scales, table, contexts, in the groups' order. A
    member other than the first has a page of NaN in place of every block that it shares."""
    rows, contexts, live = [], [], {}
    at = 1                                  # page 0: NaN
    for shared, own in groups:
        lead = list(range(at, at + shared // B))
        at += len(lead)
        live.update({p: B for p in lead})
        for i, t in enumerate(own):
            mine = list(range(at, at + -(-t // B)))
            at += len(mine)
            live.update({p: min(B, t - j * B) for j, p in enumerate(mine)})
            rows.append((lead if i == 0 else [0] * len(lead)) + mine)
            contexts.append(shared // B * B + t)
    order = torch.cat([torch.zeros(1, dtype=torch.int64), 1 + torch.randperm(at - 1, generator=gen)]).tolist()
    codes = torch.full((at, 2, H, B, D), JUNK[fmt], dtype=torch.uint8)
    scales = torch.full((at, 2, H), math.nan)
    for p, t in live.items():
        x = torch.randn(2, H, t, D, generator=gen)
        codes[order[p], :, :, :t] = (x * 100).clamp(-448, 448).to(F8).view(torch.uint8) if fmt == F8 else \
            (x * 40).round().clamp(-127, 127).to(I8).view(torch.uint8)
        scales[order[p]] = torch.exp2(torch.randint(-spread, spread + 1, (2, H), generator=gen).float()) / \
            (100 if fmt == F8 else 37)
    table = torch.zeros((len(rows), max([1] + [len(x) for x in rows])), dtype=torch.int32)
    for r, x in enumerate(rows):
        table[r, :len(x)] = torch.tensor([order[p] for p in x], dtype=torch.int32)
    return codes.view(fmt), scales, table, contexts


def run_shared(seed, groups, H, G, B, D, dtype, fmt, layout="plain", mixed=True, scale=None, stray=(), stream=None,
               q_spread=1.0):
    """`stray`: contexts of sequences behind the last group."""
    import paper_2607_02525_amd as P
    gen = torch.Generator().manual_seed(seed)
    codes, scales, table, contexts = grouped_pool(gen, list(groups) + [(0, [t]) for t in stray], B, H, D, fmt)
    n, Hq, W = len(contexts), H * G, table.shape[1]
    q, _ = rows_of(gen, (n, Hq, D), dtype, "plain", q_spread)
    sizes = [len(own) for _, own in groups]
    group_offsets = [sum(sizes[:g]) for g in range(len(sizes) + 1)]
    where = torch.randperm(n, generator=gen) if mixed else torch.arange(n)      # of the i-th member
    dq = rows_of(gen, (n, Hq, D), dtype, layout)[1]
    dq[where.cuda()] = q.cuda()
    ctx, tab = torch.empty(n, dtype=torch.int32), torch.empty_like(table)
    ctx[where], tab[where] = torch.tensor(contexts, dtype=torch.int32), table
    pool = P.KVPool(codes.cuda(), scales.cuda())
    out = torch.full_like(dq, math.nan)
    lse = torch.full((n, Hq), math.nan).cuda()
    need = P.peek_shared_decode_attention_workspace(pool, n, Hq, W, len(groups))
    ws = torch.full((max(256, need),), 0xFF, dtype=torch.uint8).cuda()
    i32 = torch.int32
    args = (pool, dq, ctx.cuda(), tab.cuda(), torch.tensor(group_offsets, dtype=i32).cuda(),
            torch.tensor([s for s, _ in groups], dtype=i32).cuda(), out, ws)
    kw = dict(members=where.to(i32).cuda() if mixed else None, lse=lse, scale=scale, stream=stream)
    torch.cuda.synchronize()
    P.peek_shared_decode_attention(*args, **kw)
    torch.cuda.synchronize()
    s, most = D ** -0.5 if scale is None else scale, R.most_of(scales, fmt)
    i = 0
    for shared, own in list(groups) + [(0, [t]) for t in stray]:
        lead = i
        for t in own:
            row = table[i].clone()
            row[:shared // B] = table[lead, :shared // B]
            k, v = R.cached(codes, scales, row, contexts[i])
            want, wl, _, spread, reach = R.attend(q[i:i + 1], k, v, s, contexts[i])
            at = int(where[i])
            near(out[at:at + 1], want, R.out_bound(want, spread, reach, dtype, contexts[i], most), f"out of member {i}")
            near(lse[at:at + 1], wl, R.lse_bound(wl, reach, D), f"lse of member {i}")
            i += 1
    return args, kw


SHARED = [
    # (shared, own tokens), kv heads, group, block, D, dtype, format
    ([(64, [5, 0, 33])], 2, 4, 16, 128, BF, F8),
    ([(64, [1]), (0, [7, 0]), (160, [16, 40])], 2, 5, 16, 128, HF, I8),
    ([(300, [300, 1, 17, 100])], 1, 8, 16, 64, BF, I8),                  # cut to 288
    ([(1040, [3] * 9), (512, [1])], 2, 3, 16, 64, HF, F8),
    ([(2048, list(range(1, 18)))], 1, 4, 32, 128, BF, F8),               # 68 rows: four tiles of 16 a workgroup
    ([(520, [9, 300, 2, 0, 44])], 2, 7, 4, 128, BF, I8),
    ([(40, [3, 4, 5]), (8, [0, 0])], 3, 1, 8, 64, HF, F8),
    ([(512, [300, 2]), (256, [513])], 1, 17, 256, 128, HF, F8),
    ([(768, [64, 65, 63])], 2, 40, 64, 64, BF, F8),
    ([(5000, [900, 20])], 1, 2, 16, 128, BF, F8),                        # many parts
    ([(15, [20, 3])], 2, 2, 16, 128, BF, I8),                            # less than a block: nothing
    ([(128, [4] * 33)], 1, 1, 128, 128, HF, I8),
    ([(64, [0, 0, 0])], 2, 4, 16, 64, BF, F8),                           # nothing of their own
    ([(1600, [3] * 45), (528, [2] * 30)], 1, 4, 16, 128, BF, F8),        # 120 to 180 rows: one or two tiles of 128
    ([(528, [3] * 45), (1040, [2] * 80)], 2, 4, 16, 64, HF, I8),
    ([(520, [1] * 20), (84, [5, 2])], 1, 16, 4, 128, HF, F8),
    ([(32 + 16 * (g % 3), [1 + g % 5] * (g % 4)) for g in range(150)], 1, 2, 16, 64, BF, I8),      # 150 groups
    ([(80, [2] * (1 + g % 3)) for g in range(70)], 1, 2, 8, 64, HF, F8),
]


@pytest.mark.parametrize("case", range(len(SHARED)))
def test_shared(case):
    print("[gpu] shared", SHARED[case], flush=True)
    run_shared(case, *SHARED[case])


@pytest.mark.parametrize("layout", ["fused", "heads first"])
def test_shared_layouts_and_order(layout):
    run_shared(20, [(96, [5, 6]), (32, [0, 40, 2])], 2, 4, 16, 128, BF, F8, layout=layout, mixed=False)


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
def test_shared_scales(scale):
    run_shared(21, [(96, [5, 6, 1])], 1, 4, 16, 64, HF, F8, scale=scale, q_spread=0.5)


def test_sequences_behind_the_last_group_and_no_groups():
    run_shared(22, [(64, [5, 6])], 2, 2, 16, 64, BF, I8, stray=(0, 17, 300))
    run_shared(23, [], 2, 2, 16, 64, BF, I8, stray=(5, 0, 600))
    run_shared(24, [(0, []), (64, [5, 6]), (640, []), (0, []), (32, [1])], 2, 2, 16, 64, BF, I8, stray=(3,))


def test_members_shorter_than_what_is_shared():
    """They read their own pages; the others what the first names."""
    import paper_2607_02525_amd as P
    gen = torch.Generator().manual_seed(9)
    codes, scales, table, contexts = grouped_pool(gen, [(128, [9, 5, 7]), (0, [40]), (0, [0])], 16, 2, 64, F8)
    n, q = 5, torch.randn(5, 4, 64, generator=gen).to(BF)
    pool = P.KVPool(codes.cuda(), scales.cuda())
    out, lse = torch.full_like(q, math.nan).cuda(), torch.full((n, 4), math.nan).cuda()
    i32 = torch.int32
    ws = torch.empty(max(256, P.peek_shared_decode_attention_workspace(pool, n, 4, table.shape[1], 1)),
                     dtype=torch.uint8).cuda()
    P.peek_shared_decode_attention(pool, q.cuda(), torch.tensor(contexts, dtype=i32).cuda(), table.cuda(),
                                   torch.tensor([0, 5], dtype=i32).cuda(), torch.tensor([128], dtype=i32).cuda(), out,
                                   ws, lse=lse)
    for r, c in enumerate(contexts):
        row = table[r].clone()
        if c >= 128:
            row[:8] = table[0, :8]
        k, v = R.cached(codes, scales, row, c)
        want, wl, _, spread, reach = R.attend(q[r:r + 1], k, v, 0.125, c)
        near(out[r:r + 1], want, R.out_bound(want, spread, reach, BF, c, R.most_of(scales, F8)), f"sequence {r}")
        near(lse[r:r + 1], wl, R.lse_bound(wl, reach, 64), f"lse of {r}")


def test_members_that_are_none_and_broken_offsets_touch_nothing():
    """Ids outside the batch, offsets and lengths out of range: the named sequences' rows are written, no others."""
    import paper_2607_02525_amd as P
    gen = torch.Generator().manual_seed(10)
    codes, scales, table, contexts = grouped_pool(gen, [(0, [40]), (0, [33]), (0, [7])], 16, 2, 64, F8)
    q = torch.randn(3, 4, 64, generator=gen).to(BF)
    pool = P.KVPool(codes.cuda(), scales.cuda())
    i32 = torch.int32
    ws = torch.empty(max(256, P.peek_shared_decode_attention_workspace(pool, 3, 4, table.shape[1], 2)),
                     dtype=torch.uint8).cuda()
    for members, offsets, shared in (([-1, 1, 7], [0, 1, 3], [16, 16]), ([99, -5, 1], [-3, 2, 900], [-1, 1 << 30])):
        out = torch.full_like(q, 7.0).cuda()
        P.peek_shared_decode_attention(pool, q.cuda(), torch.tensor(contexts, dtype=i32).cuda(), table.cuda(),
                                       torch.tensor(offsets, dtype=i32).cuda(), torch.tensor(shared, dtype=i32).cuda(),
                                       out, ws, members=torch.tensor(members, dtype=i32).cuda())
        k, v = R.cached(codes, scales, table[1], 33)
        want, _, _, spread, reach = R.attend(q[1:2], k, v, 0.125, 33)
        near(out[1:2], want, R.out_bound(want, spread, reach, BF, 33, R.most_of(scales, F8)), str(members))
        assert (out[[0, 2]] == 7.0).all()


def test_equal_inputs_give_equal_bits_and_graphs_replay():
    import paper_2607_02525_amd as P
    args, kw = run_shared(30, [(320, [5, 60, 9, 1, 2]), (64, [3, 300])], 2, 4, 16, 128, BF, F8)
    q, ctx, out, lse = args[1], args[2], args[6], kw["lse"]
    first = out.clone(), lse.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        P.peek_shared_decode_attention(*args, **kw)
    eager_out, eager_lse = torch.empty_like(out), torch.empty_like(lse)
    ws = torch.empty_like(args[7])
    for i in range(4):
        out.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        if i == 0:
            assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
        P.peek_shared_decode_attention(*args[:6], eager_out, ws, members=kw["members"], lse=eager_lse)
        torch.cuda.synchronize()
        assert torch.equal(out, eager_out) and torch.equal(lse, eager_lse)
        q.mul_(0.75)
        ctx.sub_((ctx > 330).to(torch.int32))


def test_validation_on_request(monkeypatch):
    import paper_2607_02525_amd as P
    args, kw = run_shared(32, [(96, [5, 6, 1])], 2, 4, 16, 64, HF, I8, mixed=False)
    args[3][1:, :6] = args[3][:1, :6]            # every sequence's table names what it shares
    monkeypatch.setenv("PEEK_VALIDATE", "1")
    P.peek_shared_decode_attention(*args, **kw)
    i32 = torch.int32
    for offsets, members in (([0, 4], [0, 1, 2]), ([2, 1], [0, 1, 2]), ([-1, 3], [0, 1, 2]), ([0, 3], [0, 3, 2]),
                             ([0, 3], [0, -1, 2])):
        bad = list(args)
        bad[4] = torch.tensor(offsets, dtype=i32).cuda()
        with pytest.raises(P.PeekError) as e:
            P.peek_shared_decode_attention(*bad, **{**kw, "members": torch.tensor(members, dtype=i32).cuda()})
        assert e.value.status == P.PEEK_ERR_INVALID_ARGUMENT


def test_shared_on_another_stream():
    side = torch.cuda.Stream()
    run_shared(31, [(96, [5, 6, 1])], 2, 4, 16, 64, HF, I8, stream=side)


def checked(P, groups, contexts, table, codes, scales, members=None, offsets=None, shared=None):
    """The call on these, 4 query heads to each of the pool's; returns its rows."""
    n, H, D, i32 = len(contexts), codes.shape[2], codes.shape[4], torch.int32
    gen = torch.Generator().manual_seed(n)
    q = torch.randn(n, 4 * H, D, generator=gen).to(BF)
    pool = P.KVPool(codes.cuda(), scales.cuda())
    sizes = [len(own) for _, own in groups]
    offsets = [sum(sizes[:g]) for g in range(len(sizes) + 1)] if offsets is None else offsets
    shared = [s for s, _ in groups] if shared is None else shared
    out = torch.full_like(q, 7.0).cuda()
    need = P.peek_shared_decode_attention_workspace(pool, n, 4 * H, table.shape[1], len(shared))
    ws = torch.empty(max(256, need), dtype=torch.uint8).cuda()
    P.peek_shared_decode_attention(pool, q.cuda(), torch.tensor(contexts, dtype=i32).cuda(), table.cuda(),
                                   torch.tensor(offsets, dtype=i32).cuda(), torch.tensor(shared, dtype=i32).cuda(), out,
                                   ws, members=None if members is None else torch.tensor(members, dtype=i32).cuda())
    torch.cuda.synchronize()
    return out.cpu()


def refused(P, match, *args, **kw):
    with pytest.raises(P.PeekError, match=match) as e:
        checked(P, *args, **kw)
    assert e.value.status == P.PEEK_ERR_INVALID_ARGUMENT


def test_validation_lets_pass_what_is_never_read(monkeypatch):
    """Members' own entries for what they share, whatever they are, and what the first member of a group names for tokens
    that none of it shares."""
    import paper_2607_02525_amd as P
    monkeypatch.setenv("PEEK_VALIDATE", "1")
    groups = [(96, [5, 6, 1]), (32, [3, 40]), (0, [9])]
    for B in (16, 4):
        gen = torch.Generator().manual_seed(11)
        codes, scales, table, contexts = grouped_pool(gen, groups, B, 2, 64, F8)      # (others' entries: a page of NaN)
        with_junk = checked(P, groups, contexts, table, codes, scales)
        assert with_junk.isfinite().all()
        for r in (1, 2):
            table[r, :96 // B] = -1
        table[4, :32 // B] = 1 << 30
        assert torch.equal(checked(P, groups, contexts, table, codes, scales), with_junk)
        # nobody in the group has as many tokens as are shared
        table, contexts = torch.full((2, 8), -1, dtype=torch.int32), [0, 3]
        table[1, 0] = 1
        few = scales.clone()
        few[1] = 0.5
        assert checked(P, [(8 * B, [0, 3])], contexts, table, codes, few).shape[0] == 2


def test_validation_reports_what_is_read(monkeypatch):
    """What a group shares is checked where it is read: in its first member's row, however few tokens that one has."""
    import paper_2607_02525_amd as P
    monkeypatch.setenv("PEEK_VALIDATE", "1")
    for B in (16, 4):
        groups = [(96, [5, 6, 1])]
        gen = torch.Generator().manual_seed(12)
        codes, scales, table, contexts = grouped_pool(gen, groups, B, 2, 64, I8)
        contexts[0] = 0                                        # a row of padding
        assert checked(P, groups, contexts, table, codes, scales).isfinite().all()
        for entry in (-1, len(codes), 0):                      # (page 0: scales of NaN)
            broken = table.clone()
            broken[0, 1] = entry
            refused(P, "scales" if entry == 0 else "pages", groups, contexts, broken, codes, scales)
            broken = table.clone()
            broken[2, 96 // B] = entry                         # a member's own keys
            refused(P, "scales" if entry == 0 else "pages", groups, contexts, broken, codes, scales)
        # a member with fewer tokens than are shared reads its own
        contexts[1] = 50
        refused(P, "scales", groups, contexts, table, codes, scales)
        contexts[1] = table.shape[1] * B + 1
        refused(P, "tokens", groups, contexts, table, codes, scales)
        contexts[1] = -1
        refused(P, "tokens", groups, contexts, table, codes, scales)
        contexts[1] = 102
        refused(P, "tokens", groups, contexts, table, codes, scales, shared=[-1])
        refused(P, "tokens", groups, contexts, table, codes, scales, shared=[table.shape[1] * B + 1])
        refused(P, "offsets", groups, contexts, table, codes, scales, offsets=[1, 3])
        refused(P, "twice", groups, contexts, table, codes, scales, members=[0, 1, 1])
        assert checked(P, groups, contexts, table, codes, scales, members=[0, 2, 1]).isfinite().all()
