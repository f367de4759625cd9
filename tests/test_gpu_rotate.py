"""GPU tests of peek_rotate_append and peek_kv_read against their definitions (tests/step_reference.py), and of the
first against peek_kv_append, whose codes and scales it has to leave."""
import math

import pytest

from tests import step_reference as S
from tests.test_gpu_attention import BF, F8, HF, I8, JUNK, near, rows_of

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def a_pool(gen, pages, H, B, D, fmt):
    """Pages in use: codes of all magnitudes that numbers have, scales around those of the rows to come."""
    x = torch.randn(pages, 2, H, B, D, generator=gen) * 40
    codes = x.clamp(-448, 448).to(F8) if fmt == F8 else x.round().clamp(-127, 127).to(I8)
    scales = torch.exp2(torch.randint(-3, 3, (pages, 2, H), generator=gen).float()) / (100 if fmt == F8 else 40)
    return codes, scales


ROTATE = [
    # new tokens, context, q heads, kv heads, D, block, dtype, format, rot, interleaved, norms, k_out, layout
    ([1, 1, 1], [0, 15, 16], 8, 2, 128, 16, BF, F8, 128, False, True, True, "plain"),
    ([1, 0, 5, 33], [7, 3, 0, 30], 8, 4, 128, 16, HF, I8, 128, True, True, False, "fused"),
    ([17, 2, 64], [100, 0, 1], 5, 1, 64, 16, BF, I8, 64, False, False, True, "heads first"),
    ([40, 1], [3, 1000000], 3, 3, 128, 4, HF, F8, 32, True, False, True, "fused"),
    ([70, 9], [50, 255], 2, 5, 64, 32, BF, F8, 16, False, True, True, "plain"),
    ([130, 300], [60, 0], 1, 2, 128, 64, HF, I8, 96, False, True, False, "plain"),
    ([300, 513], [200, 0], 4, 2, 64, 256, BF, F8, 48, True, True, True, "fused"),
    ([520], [1000], 0, 6, 128, 128, BF, I8, 128, False, False, False, "plain"),
    ([600, 1], [255, 256], 0, 1, 128, 256, HF, F8, 128, True, True, True, "heads first"),
    ([5, 6], [9, 12], 4, 2, 128, 8, BF, F8, 0, False, True, True, "plain"),
    ([5, 6], [9, 12], 4, 2, 64, 8, BF, F8, 0, False, False, True, "plain"),
    ([2500, 1700], [0, 333], 3, 2, 64, 16, BF, F8, 64, False, True, True, "fused"),       # four tokens a workgroup
    ([3], [2 ** 31 - 10], 2, 2, 128, 16, BF, None, 128, False, True, True, "plain"),
    ([4200, 3], [5, 100000], 2, 1, 128, 16, HF, None, 128, True, False, True, "fused"),
]


def run_rotate(seed, new, context, Hq, H, D, B, dtype, fmt, rot, inter, norms, keys, layout, in_place=False,
               magnitude=1.25, gap=2):
    import paper_2607_02525_amd as P
    gen = torch.Generator().manual_seed(seed)
    n = len(new)
    offsets = [gap]
    for t in new:
        offsets.append(offsets[-1] + t)
    T = offsets[-1] + gap                  # rows of no sequence before and after
    q, dq = rows_of(gen, (T, max(Hq, 1), D), dtype, layout, 1.5)
    k, dk = rows_of(gen, (T, H, D), dtype, layout, 2.0)
    v, dv = rows_of(gen, (T, H, D), dtype, layout)
    freq = torch.tensor([10000.0 ** (-2 * i / rot) for i in range(rot // 2)], dtype=torch.float64) if rot else None
    qn, kn = ((1 + 0.3 * torch.randn(D, generator=gen)).to(dtype) if norms else None for _ in range(2))
    eps = 1e-5
    q_out, k_out = (dq, dk) if in_place else (torch.full_like(dq, math.nan), torch.full_like(dk, math.nan))
    before = q_out.clone(), k_out.clone()
    pool = table = None
    if fmt is not None:
        width = max(-(-(c + t) // B) for c, t in zip(context, new))
        blocks = [(r, b) for r in range(n) for b in range(context[r] // B, -(-(context[r] + new[r]) // B))]
        codes, scales = a_pool(gen, len(blocks) + 2, H, B, D, fmt)
        table = torch.zeros((n, max(1, width)), dtype=torch.int32)
        for (r, b), p in zip(blocks, torch.randperm(len(blocks) + 2, generator=gen).tolist()):
            table[r, b] = p
        pool, other = (P.KVPool(codes.cuda(), scales.cuda()) for _ in range(2))
        table = table.cuda()
    at = torch.tensor(offsets, dtype=torch.int64).cuda()
    ctx = torch.tensor(context, dtype=torch.int32).cuda()
    cuda = [x if x is None else x.cuda() for x in (freq, qn, kn)]
    torch.cuda.synchronize()
    P.peek_rotate_append(dq if Hq else None, dk, dv if pool else None, at, ctx, cuda[0], q_out if Hq else None,
                         k_out=k_out if keys else None, pool=pool, block_table=table, interleaved=inter,
                         magnitude=magnitude, q_norm=cuda[1], k_norm=cuda[2], eps=eps)
    torch.cuda.synchronize()
    live = S.positions(offsets, context)
    some = live if len(live) < 400 else live[:150] + live[-150:] + live[150:-150:29]
    for x, got, norm, on in ((q, q_out, qn, Hq > 0), (k, k_out, kn, keys)):
        if not on:
            continue
        for t, p in some:
            want, size = S.rotate(x[t], p, None if freq is None else freq.tolist(), inter, magnitude, norm, eps)
            near(got[t], want, S.rotate_bound(want, size, dtype, D, p), f"token {t} at {p}")
        rest = sorted(set(range(T)) - {t for t, _ in live})
        old = before[0 if x is q else 1]
        assert torch.equal(got[rest].view(torch.int16), old[rest].view(torch.int16)), "rows of no sequence"
    if pool is not None:
        rotated = k_out
        if not keys:                        # the same rows without a pool
            rotated = torch.full_like(dk, math.nan)
            P.peek_rotate_append(None, dk, None, at, ctx, cuda[0], None, k_out=rotated, interleaved=inter,
                                 magnitude=magnitude, k_norm=cuda[2], eps=eps)
        P.peek_kv_append(other, rotated, dv, at, ctx, table)
        torch.cuda.synchronize()
        assert torch.equal(pool.pages.view(torch.uint8), other.pages.view(torch.uint8)), "codes"
        assert torch.equal(pool.scales.view(torch.int32), other.scales.view(torch.int32)), "scales"


@pytest.mark.parametrize("case", range(len(ROTATE)))
def test_rotate(case):
    print("[gpu] rotate", ROTATE[case], flush=True)
    run_rotate(case, *ROTATE[case])


@pytest.mark.parametrize("case", [0, 2, 4, 6, 8, 11, 13])
def test_rotate_in_place(case):
    print("[gpu] rotate in place", ROTATE[case], flush=True)
    run_rotate(case, *ROTATE[case], in_place=True)


@pytest.mark.parametrize("inter", [False, True])
def test_far_positions_keep_their_angles(inter):
    """Positions close to 2^31 with frequencies up to a radian: 32 bits would lose the whole angle."""
    run_rotate(5, [4, 4], [2 ** 31 - 4, 2 ** 31 - 2000], 2, 1, 128, 16, HF, None, 128, inter, False, True, "plain")


def test_rotate_infinities_and_nan_stay_in_their_head():
    import paper_2607_02525_amd as P
    gen = torch.Generator().manual_seed(3)
    q = torch.randn(4, 6, 128, generator=gen).to(BF)
    q[1, 2, 5], q[2, 0, 7], q[3, 1, 70] = math.inf, math.nan, -math.inf
    freq = torch.tensor([10000.0 ** (-i / 64) for i in range(64)], dtype=torch.float64)
    out = torch.empty_like(q).cuda()
    clean = torch.where(q.isfinite(), q, torch.zeros_like(q))
    ref = torch.empty_like(out)
    at, ctx = torch.tensor([0, 4]).cuda(), torch.tensor([9], dtype=torch.int32).cuda()
    for x, y in ((q, out), (clean, ref)):
        P.peek_rotate_append(None, x.cuda(), None, at, ctx, freq.cuda(), None, k_out=y)
    a, b = out.cpu(), ref.cpu()
    touched = torch.zeros_like(q, dtype=torch.bool)
    for t, h, i in ((1, 2, 5), (2, 0, 7), (3, 1, 6)):
        touched[t, h, i] = touched[t, h, i + 64] = True
    assert torch.equal(a[~touched], b[~touched])
    assert not a[1, 2, 5].isfinite() and a[2, 0, 7].isnan()


def test_blocks_that_have_no_page_are_left_out_and_their_rows_are_not():
    """A page id outside the pool, and tokens past the table: nothing of the pool changes, k_out has its rows."""
    import paper_2607_02525_amd as P
    gen = torch.Generator().manual_seed(8)
    codes, scales = a_pool(gen, 3, 2, 16, 64, I8)
    pool = P.KVPool(codes.cuda(), scales.cuda())
    k, v = (torch.randn(60, 2, 64, generator=gen).to(BF).cuda() for _ in range(2))
    at, ctx = torch.tensor([0, 20, 60]).cuda(), torch.tensor([0, 16], dtype=torch.int32).cuda()
    table = torch.tensor([[-1, 3], [0, 77]], dtype=torch.int32).cuda()
    freq = torch.tensor([1.0] * 8, dtype=torch.float64).cuda()
    out, want = (torch.full_like(k, math.nan) for _ in range(2))
    P.peek_rotate_append(None, k, v, at, ctx, freq, None, k_out=out, pool=pool, block_table=table)
    P.peek_rotate_append(None, k, None, at, ctx, freq, None, k_out=want)
    assert torch.equal(out, want) and not out.isnan().any()
    assert torch.equal(pool.pages.cpu(), codes) and torch.equal(pool.scales.cpu(), scales)


# -------------------------------------------------------------------- read
READ = [
    ([5, 0, 16, 17], [0, 3, 16, 30], 2, 16, 128, BF, F8, "plain"),
    ([1], [0], 1, 16, 64, HF, I8, "plain"),
    ([300, 1], [7, 255], 3, 256, 64, BF, I8, "fused"),
    ([33, 70], [2, 0], 5, 4, 128, HF, F8, "heads first"),
    ([129], [64], 2, 64, 128, HF, I8, "fused"),
]


@pytest.mark.parametrize("case", range(len(READ)))
def test_read(case):
    import paper_2607_02525_amd as P
    new, first, H, B, D, dtype, fmt, layout = READ[case]
    print("[gpu] read", READ[case], flush=True)
    gen = torch.Generator().manual_seed(case)
    blocks = [-(-(f + t) // B) for f, t in zip(first, new)]
    codes, scales = a_pool(gen, sum(blocks) + 1, H, B, D, fmt)
    raw = codes.view(torch.uint8)
    raw[0, :, :, 0, :3] = JUNK[fmt]
    table = torch.zeros((len(new), max(blocks)), dtype=torch.int32)
    ids = torch.randperm(sum(blocks) + 1, generator=gen).tolist()
    for r, b in enumerate(blocks):
        for i in range(b):
            table[r, i] = ids.pop()
    offsets = [1]
    for t in new:
        offsets.append(offsets[-1] + t)
    T = offsets[-1] + 2
    outs = [torch.full_like(rows_of(gen, (T, H, D), dtype, layout)[1], 7.0) for _ in range(2)]
    P.peek_kv_read(P.KVPool(codes.cuda(), scales.cuda()), torch.tensor(offsets).cuda(),
                   torch.tensor(first, dtype=torch.int32).cuda(), table.cuda(), *outs)
    torch.cuda.synchronize()
    for part, out in enumerate(outs):
        want = torch.full((T, H, D), 7.0, dtype=dtype)
        for r, t in enumerate(new):
            for i in range(t):
                p = int(table[r, (first[r] + i) // B])
                x = codes[p, part, :, (first[r] + i) % B].float() * scales[p, part][:, None]
                want[offsets[r] + i] = x.to(dtype)
        a, b = out.cpu(), want
        assert torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(), b.nan_to_num())


def test_read_past_the_table_leaves_rows_alone():
    import paper_2607_02525_amd as P
    gen = torch.Generator().manual_seed(1)
    codes, scales = a_pool(gen, 2, 1, 16, 64, F8)
    outs = [torch.full((40, 1, 64), 5.0, dtype=BF).cuda() for _ in range(2)]
    table = torch.tensor([[1, 0]], dtype=torch.int32).cuda()
    P.peek_kv_read(P.KVPool(codes.cuda(), scales.cuda()), torch.tensor([0, 40]).cuda(),
                   torch.tensor([-3], dtype=torch.int32).cuda(), table, *outs)
    for part, out in enumerate(outs):
        want = (codes[[1, 0], part].float() * scales[[1, 0], part][..., None, None]).to(BF)
        assert torch.equal(out[:32].cpu(), want.transpose(1, 2).reshape(32, 1, 64))
        assert (out[32:] == 5.0).all()


def test_rotation_captured_and_replayed():
    """A graph of rotation, append and read, replayed with other inputs in place, against eager calls."""
    import paper_2607_02525_amd as P
    gen = torch.Generator().manual_seed(4)
    n, H, Hq, D, B = 3, 2, 4, 128, 16
    codes, scales = a_pool(gen, 12, H, B, D, F8)
    pool, other = (P.KVPool(codes.cuda(), scales.cuda()) for _ in range(2))
    at = torch.arange(n + 1, dtype=torch.int64).cuda()
    ctx = torch.tensor([0, 14, 30], dtype=torch.int32).cuda()
    table = torch.arange(12, dtype=torch.int32).view(3, 4).cuda()
    freq = torch.tensor([10000.0 ** (-i / 64) for i in range(64)], dtype=torch.float64).cuda()
    q, k, v = (torch.zeros(n, h, D, dtype=BF).cuda() for h in (Hq, H, H))
    outs = [torch.zeros_like(x) for x in (q, k, k, k)]
    eager = [torch.zeros_like(x) for x in outs]

    def step(pool, o):
        P.peek_rotate_append(q, k, v, at, ctx, freq, o[0], k_out=o[1], pool=pool, block_table=table)
        P.peek_kv_read(pool, at, ctx, table, o[2], o[3])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(pool, outs)
    for i in range(4):
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, generator=gen).to(BF))
        ctx += 1
        graph.replay()
        step(other, eager)
        torch.cuda.synchronize()
        for a, b in zip(outs, eager):
            assert torch.equal(a, b)
        assert torch.equal(pool.pages.view(torch.uint8), other.pages.view(torch.uint8))


@pytest.mark.parametrize("layout", ["plain", "fused", "heads first"])
def test_queries_alone(layout):
    """Without keys: as beside them."""
    import paper_2607_02525_amd as P
    gen = torch.Generator().manual_seed(12)
    T, Hq, D = 9, 6, 128
    q, dq = rows_of(gen, (T, Hq, D), BF, layout)
    _, dk = rows_of(gen, (T, 2, D), BF, "plain")
    at, ctx = torch.tensor([1, 4, 8]).cuda(), torch.tensor([7, 0], dtype=torch.int32).cuda()
    freq = torch.tensor([10000.0 ** (-i / 64) for i in range(64)], dtype=torch.float64).cuda()
    norm = (1 + 0.3 * torch.randn(D, generator=gen)).to(BF).cuda()
    alone, beside = torch.full_like(dq, math.nan), torch.full_like(dq, math.nan)
    P.peek_rotate_append(dq, None, None, at, ctx, freq, alone, q_norm=norm)
    P.peek_rotate_append(dq, dk, None, at, ctx, freq, beside, k_out=torch.empty_like(dk), q_norm=norm)
    assert torch.equal(alone.view(torch.int16), beside.view(torch.int16))
    for t, p in S.positions([1, 4, 8], [7, 0]):
        want, size = S.rotate(q[t], p, freq.tolist(), False, 1.0, norm.cpu(), 1e-6)
        near(alone[t], want, S.rotate_bound(want, size, BF, D, p), f"token {t} at {p}")
