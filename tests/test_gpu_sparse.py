"""GPU tests of peek_kv_bounds, peek_block_select and peek_sparse_decode_attention against their definitions: whole
numbers for the first two (tests/step_reference.py), 64 bits for the attention (tests/kv_reference.py)."""
import math

import numpy as np
import pytest

from tests import kv_reference as R
from tests import step_reference as S
from tests.test_gpu_attention import BF, F8, HF, I8, JUNK, make_pool, near, rows_of

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def ints(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def all_bounds(codes, scales, table, contexts, first=None):
    """[P, H, 2, D] int8; 99 where no block was looked at."""
    P_, _, H, B, D = codes.shape
    out = np.full((P_, H, 2, D), 99, np.int8)
    for r, c in enumerate(contexts):
        for b in range((0 if first is None else max(0, first[r])) // B, -(-c // B)):
            p = int(table[r, b])
            hi, lo = S.bounds(codes, scales, p, min(B, c - b * B))
            out[p, :, 0], out[p, :, 1] = hi, lo
    return torch.from_numpy(out)


BOUNDS = [
    ([0, 1, 15, 16, 17, 300], 2, 16, 128, F8, None),
    ([5, 4, 9, 0], 3, 4, 64, I8, None),
    ([700, 31], 1, 256, 128, I8, None),
    ([64, 65, 200], 5, 64, 64, F8, [63, 65, 100]),
    ([33, 8, 500], 2, 8, 128, F8, [32, 0, -4]),
    ([2000, 128], 1, 128, 64, I8, [1999, 500]),
    ([90], 2, 32, 128, F8, [89]),
]


@pytest.mark.parametrize("case", range(len(BOUNDS)))
def test_bounds(case):
    import paper_2607_02525_amd as P
    contexts, H, B, D, fmt, first = BOUNDS[case]
    print("[gpu] bounds", BOUNDS[case], flush=True)
    gen = torch.Generator().manual_seed(case)
    codes, scales, table = make_pool(gen, contexts, H, B, D, fmt)
    raw = codes.view(torch.uint8)
    raw[int(table[0, 0]), 0, 0, 0, 3], raw[int(table[0, 0]), 0, 0, 0, 4] = 0x7F, 0xFF      # NaN of both signs (127, -1)
    raw[int(table[-1, 0]), 0, 0, 0, 0] = 0x80                                              # -0, or -128
    scales[int(table[0, 0]), 0] *= -1                                                      # keys of a negative scale
    got = torch.full((codes.shape[0], H, 2, D), 99, dtype=torch.int8).cuda()
    P.peek_kv_bounds(P.KVPool(codes.cuda(), scales.cuda()), None if first is None else ints(first), ints(contexts),
                     table.cuda(), got)
    assert torch.equal(got.cpu(), all_bounds(codes, scales, table, contexts, first))


def test_every_float8_code_is_bounded():
    import paper_2607_02525_amd as P
    codes = torch.zeros(4, 2, 1, 4, 64, dtype=torch.uint8)
    codes[:, 0, 0, 0] = torch.arange(256, dtype=torch.uint8).view(4, 64)
    codes = codes.view(F8)
    scales, table = torch.ones(4, 2, 1), torch.arange(4, dtype=torch.int32).view(4, 1)
    got = torch.empty(4, 1, 2, 64, dtype=torch.int8).cuda()
    P.peek_kv_bounds(P.KVPool(codes.cuda(), scales.cuda()), None, ints([1] * 4), table.cuda(), got)
    assert torch.equal(got.cpu(), all_bounds(codes, scales, table, [1] * 4))


SELECT = [
    # contexts, keep, sink, recent, kv heads, group, block, D, dtype, format
    ([0, 1, 16, 17, 100, 160, 161, 400], 10, 1, 2, 2, 4, 16, 128, BF, F8),
    ([1000, 999, 63], 6, 1, 1, 1, 1, 4, 64, HF, I8),
    ([3000, 70], 33, 0, 1, 3, 5, 16, 64, BF, I8),
    ([2100, 640], 8, 3, 5, 2, 17, 64, 128, HF, F8),            # sink and recent are all of it
    ([5000], 100, 2, 2, 1, 40, 8, 128, BF, F8),
    ([9000, 4100, 8192], 64, 1, 2, 2, 8, 16, 128, BF, F8),
    ([4000], 1, 0, 1, 2, 2, 32, 64, BF, I8),
    ([40000, 256], 77, 1, 2, 1, 16, 4, 64, HF, F8),            # 10000 blocks
]


def select(P, pool, bounds, q, contexts, table, keep, sink, recent):
    n, H = len(contexts), pool.kv_heads
    ctx_out = torch.full((n, H), -7, dtype=torch.int32).cuda()
    table_out = torch.full((n, H, keep), -7, dtype=torch.int32).cuda()
    ws = torch.full((max(256, P.peek_block_select_workspace(pool, n, table.shape[1])),), 0xFF, dtype=torch.uint8).cuda()
    P.peek_block_select(pool, bounds, q, ints(contexts), table.cuda(), sink, recent, ctx_out, table_out, ws)
    torch.cuda.synchronize()
    return ctx_out, table_out


def chosen(codes, scales, bounds, q, contexts, table, keep, sink, recent):
    """By the definition: table_out and context_out, and the blocks."""
    n, H, B = len(contexts), codes.shape[2], codes.shape[3]
    G = q.shape[1] // H
    t_out, c_out = torch.full((n, H, keep), -1, dtype=torch.int32), torch.zeros(n, H, dtype=torch.int32)
    for r, c in enumerate(contexts):
        nb = -(-c // B)
        ids = table[r, :nb].long()
        for h in range(H):
            x = bounds[ids, h].numpy().astype(np.int64)
            score = S.scores(q[r, h * G:(h + 1) * G], x[:, 0], x[:, 1], scales[ids, 0, h].numpy(), codes.dtype) \
                if nb else np.zeros(0)
            stay = S.choose(score, nb, keep, sink, recent)
            t_out[r, h, :len(stay)] = table[r, stay]
            c_out[r, h] = c - (nb - len(stay)) * B
    return t_out, c_out


@pytest.mark.parametrize("case", range(len(SELECT)))
def test_select_and_attend(case):
    import paper_2607_02525_amd as P
    contexts, keep, sink, recent, H, G, B, D, dtype, fmt = SELECT[case]
    print("[gpu] select", SELECT[case], flush=True)
    gen = torch.Generator().manual_seed(case)
    codes, scales, table = make_pool(gen, contexts, H, B, D, fmt)
    n, Hq = len(contexts), H * G
    q, dq = rows_of(gen, (n, Hq, D), dtype, ["plain", "fused", "heads first"][case % 3], 1.5)
    pool = P.KVPool(codes.cuda(), scales.cuda())
    bounds = torch.full((codes.shape[0], H, 2, D), 99, dtype=torch.int8).cuda()
    P.peek_kv_bounds(pool, None, ints(contexts), table.cuda(), bounds)
    ctx_out, table_out = select(P, pool, bounds, dq, contexts, table, keep, sink, recent)
    t, c = chosen(codes, scales, bounds.cpu(), q, contexts, table, keep, sink, recent)
    assert torch.equal(ctx_out.cpu(), c)
    assert torch.equal(table_out.cpu(), t)
    out, lse = torch.full_like(dq, math.nan), torch.full((n, Hq), math.nan).cuda()
    ws = torch.full((max(256, P.peek_sparse_decode_attention_workspace(pool, n, Hq, keep)),), 0xFF,
                    dtype=torch.uint8).cuda()
    P.peek_sparse_decode_attention(pool, dq, ctx_out, table_out, out, ws, lse=lse)
    torch.cuda.synchronize()
    most = R.most_of(scales, fmt)
    for r in range(n):
        for h in range(H):
            tokens = int(c[r, h])
            k, v = R.cached(codes[:, :, h:h + 1], scales[:, :, h:h + 1], t[r, h], tokens)
            rows = slice(h * G, (h + 1) * G)
            want, wl, _, spread, reach = R.attend(q[r:r + 1, rows], k, v, D ** -0.5, tokens)
            near(out[r:r + 1, rows], want, R.out_bound(want, spread, reach, dtype, tokens, most), f"out {r} {h}")
            near(lse[r:r + 1, rows], wl, R.lse_bound(wl, reach, D), f"lse {r} {h}")


def by_hand(fmt, scales_of, q, keep, sink=0, recent=1, D=64, B=4):
    """Blocks whose keys are all 8 (code), with these scales: what is kept."""
    import paper_2607_02525_amd as P
    nb = len(scales_of)
    codes = torch.zeros(nb, 2, 1, B, D, dtype=torch.uint8)
    codes[:] = torch.tensor([8.0]).to(fmt).view(torch.uint8)
    scales = torch.ones(nb, 2, 1)
    scales[:, 0, 0] = torch.tensor(scales_of)
    codes = codes.view(fmt)
    table = torch.arange(nb, dtype=torch.int32).view(1, nb)
    pool = P.KVPool(codes.cuda(), scales.cuda())
    bounds = torch.empty(nb, 1, 2, D, dtype=torch.int8).cuda()
    P.peek_kv_bounds(pool, None, ints([nb * B]), table.cuda(), bounds)
    ctx, t = select(P, pool, bounds, q.cuda(), [nb * B], table, keep, sink, recent)
    want, c = chosen(codes, scales, bounds.cpu(), q, [nb * B], table, keep, sink, recent)
    assert torch.equal(t.cpu(), want) and torch.equal(ctx.cpu(), c)
    return t.cpu().flatten().tolist()


@pytest.mark.parametrize("fmt", [F8, I8], ids=["f8", "i8"])
def test_ties_signs_and_values_that_are_no_numbers(fmt):
    ones = torch.ones(1, 1, 64).to(BF)
    assert by_hand(fmt, [1.0] * 9, ones, 4) == [0, 1, 2, 8]                       # equal scores by position
    assert by_hand(fmt, [1.0] * 9, torch.zeros(1, 3, 64).to(BF), 4) == [0, 1, 2, 8]
    assert by_hand(fmt, [1.0, 3.0, 2.0, 3.0, 1.0], ones, 3) == [1, 3, 4]
    assert by_hand(fmt, [1.0, 3.0, 2.0, 3.0, 1.0], -ones, 3) == [0, 2, 4]          # below 0: the smaller scale
    assert by_hand(fmt, [1.0, math.nan, 2.0, 3.0, 1.0, math.nan, 0.5], ones, 4) == [1, 3, 5, 6]
    assert by_hand(fmt, [1.0, -3.0, 2.0, -1.0, 1.0], ones, 3) == [0, 2, 4]         # keys of a negative scale
    assert by_hand(fmt, [1.0, -3.0, 2.0, -1.0, 1.0], -ones, 3) == [1, 3, 4]
    assert by_hand(fmt, [0.0, -0.0, 0.0, 1.0], -ones, 3) == [0, 1, 3]              # -0 and 0 are equal
    wild = torch.ones(1, 2, 64)
    wild[0, 0, 5], wild[0, 1, 9], wild[0, 0, 6] = math.inf, math.nan, -math.inf
    by_hand(fmt, [1.0, 3.0, 2.0, 3.0, 1.0], wild.to(BF), 3)
    by_hand(fmt, [1e38, 3.0, 2e38, 3.0, 1.0, 1e-38], ones * 1e30, 4)               # scores beyond float32: equal
    by_hand(fmt, [1.0, 3.0, 2.0, 3.0, 1.0], (ones * 2.0 ** -120), 3)
    by_hand(fmt, [1.0, 3.0, 2.0, 3.0, 1.0], torch.full((1, 1, 64), 2.0 ** -24).half(), 3)      # float16's least
    by_hand(fmt, [2.0 ** -i for i in range(300)], ones, 100, sink=3, recent=4)


def test_page_ids_outside_the_pool_are_never_followed():
    """They read as page 0, and are handed on as they are."""
    import paper_2607_02525_amd as P
    gen = torch.Generator().manual_seed(2)
    codes, scales, table = make_pool(gen, [400], 2, 16, 64, F8)
    bounds = torch.zeros(codes.shape[0], 2, 2, 64, dtype=torch.int8).cuda()
    pool = P.KVPool(codes.cuda(), scales.cuda())
    P.peek_kv_bounds(pool, None, ints([400]), table.cuda(), bounds)
    broken = table.clone()
    broken[0, 5], broken[0, 7], broken[0, 24] = -1, 1 << 30, 12345
    as_read = torch.where((broken < 0) | (broken >= codes.shape[0]), torch.zeros_like(broken), broken)
    q = torch.randn(1, 4, 64, generator=gen).to(BF)
    ctx, t = select(P, pool, bounds, q.cuda(), [400], broken, 20, 8, 2)
    want, c = chosen(codes, scales, bounds.cpu(), q, [400], as_read, 20, 8, 2)
    got = t.cpu()
    assert torch.equal(torch.where((got < 0) | (got >= codes.shape[0]), torch.zeros_like(got), got), want)
    assert (got == -1).any() and (got == 1 << 30).any() and (got == 12345).any()


def test_a_step_of_everything_captured_and_replayed():
    """Rotation and append, bounds, choice, attention over the chosen and over all blocks, as a decoding step makes
    them; with every block kept, the attentions agree."""
    import paper_2607_02525_amd as P
    gen = torch.Generator().manual_seed(12)
    n, H, G, D, B, width = 4, 2, 4, 128, 16, 24
    contexts = [100, 250, 3, 380]
    codes, scales, _ = make_pool(gen, [width * B] * n, H, B, D, F8, spare=0)
    table = torch.randperm(n * width, generator=gen).to(torch.int32).view(n, width).cuda()
    at, ctx = torch.arange(n + 1).cuda(), ints(contexts)
    freq = torch.from_numpy(P.peek_rotary_frequencies(D, 500000.0, P.PEEK_ROTARY_TURNS, 8.0, 8192.0)).cuda()
    q, k, v = (torch.zeros(n, h, D, dtype=BF).cuda() for h in (H * G, H, H))

    class Side:
        def __init__(self, keep):
            self.pool = P.KVPool(codes.cuda(), scales.cuda())
            self.keep, self.q = keep, torch.zeros_like(q)
            self.bounds = torch.zeros(n * width, H, 2, D, dtype=torch.int8).cuda()
            self.ctx, self.table = ints([[0] * H] * n), torch.zeros(n, H, keep, dtype=torch.int32).cuda()
            self.out, self.dense, self.shared = (torch.zeros_like(q) for _ in range(3))
            need = max(P.peek_block_select_workspace(self.pool, n, width),
                       P.peek_sparse_decode_attention_workspace(self.pool, n, H * G, keep),
                       P.peek_decode_attention_workspace(self.pool, n, H * G, width),
                       P.peek_shared_decode_attention_workspace(self.pool, n, H * G, width, n))
            self.ws = torch.empty(max(256, need), dtype=torch.uint8).cuda()
            self.after = torch.zeros_like(ctx)
            self.groups = torch.arange(n + 1, dtype=torch.int32).cuda()
            P.peek_kv_bounds(self.pool, None, ctx, table, self.bounds)

        def step(self):
            P.peek_rotate_append(q, k, v, at, ctx, freq, self.q, pool=self.pool, block_table=table)
            torch.add(ctx, 1, out=self.after)
            P.peek_kv_bounds(self.pool, ctx, self.after, table, self.bounds)
            P.peek_block_select(self.pool, self.bounds, self.q, self.after, table, 1, 2, self.ctx, self.table, self.ws)
            P.peek_sparse_decode_attention(self.pool, self.q, self.ctx, self.table, self.out, self.ws)
            P.peek_decode_attention(self.pool, self.q, self.after, table, self.dense, self.ws)
            P.peek_shared_decode_attention(self.pool, self.q, self.after, table, self.groups, self.after, self.shared,
                                           self.ws)

    for keep in (6, width):
        ctx.copy_(ints(contexts))
        a, b = Side(keep), Side(keep)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            a.step()
        for i in range(3):
            for x in (q, k, v):
                x.copy_(torch.randn(x.shape, generator=gen).to(BF))
            graph.replay()
            b.step()
            torch.cuda.synchronize()
            for name in ("q", "bounds", "ctx", "table", "out", "dense", "shared"):
                assert torch.equal(getattr(a, name), getattr(b, name)), name
            # both are off from the exact result by out_bound at most, whose largest part is two roundings
            for x in (a.shared, a.out if keep == width else a.shared):
                assert (x.float() - a.dense.float()).abs().max() <= 2 * 3 * 2.0 ** -8 * a.dense.float().abs().max() + 0.05
            ctx += 1


@pytest.mark.parametrize("fmt", [F8, I8], ids=["f8", "i8"])
def test_scores_too_small_for_32_bits_are_equal_whatever_their_sign(fmt):
    """Queries of 2^-120 and scales of 2^-60: every score is 0, also that of a key against the query."""
    import paper_2607_02525_amd as P
    nb, B, D, keep = 12, 4, 64, 5
    codes = torch.empty(nb, 2, 1, B, D, dtype=torch.uint8)
    for b in range(nb):
        codes[b] = torch.tensor([-8.0 if b % 2 == 0 else 8.0]).to(fmt).view(torch.uint8)
    codes, scales = codes.view(fmt), torch.full((nb, 2, 1), 2.0 ** -60)
    q, table = torch.full((1, 1, D), 2.0 ** -120, dtype=BF), torch.arange(nb, dtype=torch.int32).view(1, nb)
    pool = P.KVPool(codes.cuda(), scales.cuda())
    bounds = torch.empty(nb, 1, 2, D, dtype=torch.int8).cuda()
    P.peek_kv_bounds(pool, None, ints([nb * B]), table.cuda(), bounds)
    _, t = select(P, pool, bounds, q.cuda(), [nb * B], table, keep, 0, 1)
    want, _ = chosen(codes, scales, bounds.cpu(), q, [nb * B], table, keep, 0, 1)
    assert want.flatten().tolist() == [0, 1, 2, 3, nb - 1]
    assert torch.equal(t.cpu(), want)


def test_bounds_of_no_page_are_left_out():
    """A page id outside the pool: page 0 is another sequence's, whose bounds stay."""
    import paper_2607_02525_amd as P
    gen = torch.Generator().manual_seed(5)
    codes, scales, _ = make_pool(gen, [64], 2, 16, 64, I8, spare=0)
    table = torch.tensor([[1, -1, 3, 4]], dtype=torch.int32)
    bounds = torch.full((4, 2, 2, 64), 99, dtype=torch.int8).cuda()
    P.peek_kv_bounds(P.KVPool(codes.cuda(), scales.cuda()), None, ints([64]), table.cuda(), bounds)
    got = bounds.cpu()
    assert (got[[0, 2]] == 99).all(), "pages that the sequence does not name"
    for p in (1, 3):
        hi, lo = S.bounds(codes, scales, p, 16)
        assert torch.equal(got[p], torch.from_numpy(np.stack([hi, lo], 1).astype(np.int8)))
