"""GPU tests of the calls around a decode step at the ends of their ranges: sequences close to 2^31 tokens (every block
but the last is one page, so that the sums over all of it are known), more heads than the device has places for
workgroups, and rows that must not reach each other."""
import math

import pytest

from tests import kv_reference as R
from tests.test_gpu_attention import BF, F8, HF, I8, JUNK, near

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
I32 = torch.int32


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def long_pool(P, B, fmt, tokens, D):
    last, live = (tokens - 1) // B, (tokens - 1) % B + 1
    codes = torch.zeros(2, 2, 1, B, D)
    codes[0, 1] = 3
    codes[1, 0, 0, :, 0] = 40
    codes[1, 1, 0] = (torch.arange(B) % 8 + 1)[:, None].float()
    codes = codes.to(fmt)
    codes.view(torch.uint8)[1, :, :, live:] = JUNK[fmt]
    return P.KVPool(codes.cuda(), torch.ones(2, 2, 1).cuda()), last, live


@pytest.mark.parametrize("B,fmt,tokens,G", [(256, I8, 2 ** 31 - 256, 2), (256, F8, 2 ** 31 - 256 - 100, 80),
                                            (4, F8, 2 ** 31 - 5, 80), (16, I8, 2 ** 31 - 16 - 3, 2)])
def test_shared_lengths_close_to_the_end_of_32_bits(B, fmt, tokens, G):
    import paper_2607_02525_amd as P
    print("[gpu] shared long", B, fmt, tokens, G, flush=True)
    D, W, n = 64, (2 ** 31 - 1) // B, 2
    pool, last, live = long_pool(P, B, fmt, tokens, D)
    table = torch.zeros(n, W, dtype=I32, device="cuda")
    table[:, last] = 1
    q = torch.zeros(n, G, D, dtype=BF)
    q[:, 0, 0] = 1                        # this head looks at the last block, the others at all tokens alike
    out, lse = torch.empty(n, G, D, dtype=BF).cuda(), torch.empty(n, G).cuda()
    ws = torch.empty(max(256, P.peek_shared_decode_attention_workspace(pool, n, G, W, 1)), dtype=torch.uint8).cuda()
    P.peek_shared_decode_attention(pool, q.cuda(), torch.tensor([tokens] * n, dtype=I32).cuda(), table,
                                   torch.tensor([0, n], dtype=I32).cuda(), torch.tensor([tokens], dtype=I32).cuda(), out,
                                   ws, scale=1.0, lse=lse)
    torch.cuda.synchronize()
    mean = (torch.arange(live) % 8 + 1).double().mean()
    many, few = tokens - live, live * math.exp(40)
    sums = torch.tensor([many + few] + [tokens] * (G - 1)).double()
    value = torch.tensor([3 * many + few * mean] + [3 * many + live * mean] * (G - 1)).double() / sums
    near(out, value[None, :, None].expand(n, G, D), 2.0 ** -7 * value[None, :, None], "out")
    near(lse, sums.log()[None].expand(n, G), R.lse_bound(sums.log()[None], 40.0, D), "lse")


def test_choice_close_to_the_end_of_32_bits():
    """8.4 million blocks, of which all but the last are alike: these go by position."""
    import paper_2607_02525_amd as P
    B, D, tokens, keep = 256, 64, 2 ** 31 - 256 - 100, 5
    W = (2 ** 31 - 1) // B
    pool, last, live = long_pool(P, B, I8, tokens, D)
    table = torch.zeros(1, W, dtype=I32, device="cuda")
    table[0, last] = 1
    held = torch.tensor([tokens], dtype=I32).cuda()
    bounds = torch.full((2, 1, 2, D), 99, dtype=torch.int8).cuda()
    P.peek_kv_bounds(pool, None, held, table, bounds)
    want = torch.zeros(2, 1, 2, D, dtype=torch.int8)
    want[1, 0, :, 0] = 40
    assert torch.equal(bounds.cpu(), want)
    q = torch.zeros(1, 1, D, dtype=BF)
    q[0, 0, 0] = 1
    ctx, kept = torch.empty(1, 1, dtype=I32).cuda(), torch.empty(1, 1, keep, dtype=I32).cuda()
    ws = torch.empty(P.peek_block_select_workspace(pool, 1, W), dtype=torch.uint8).cuda()
    P.peek_block_select(pool, bounds, q.cuda(), held, table, 0, 1, ctx, kept, ws)
    assert kept.flatten().tolist() == [0, 0, 0, 0, 1] and int(ctx) == 4 * B + live


@pytest.mark.parametrize("H,G,B", [(600, 1, 16), (1024, 3, 16), (600, 2, 8)])
def test_more_heads_than_pieces(H, G, B):
    """One piece of the shared keys to a head, which goes through all groups' tiles."""
    import paper_2607_02525_amd as P
    from tests.test_gpu_shared import run_shared
    print("[gpu] heads", H, G, B, flush=True)
    run_shared(H, [(32, [1, 0]), (16, [3])], H, G, B, 64, HF, F8)


@pytest.mark.parametrize("groups,G", [([(64, [5, 3, 9])], 4), ([(128, [2] * 20)], 8)])
def test_a_member_of_nan_reaches_no_other(groups, G):
    """Queries of infinities and NaN beside others in the same tiles: the others' bits are as without them."""
    import paper_2607_02525_amd as P
    from tests.test_gpu_shared import run_shared
    args, kw = run_shared(3, groups, 2, G, 16, 128, BF, F8, mixed=False)
    clean = args[6].clone()
    q = args[1]
    q[1] = math.nan
    q[2, 0, 0], q[2, 1, 3] = math.inf, -math.inf
    P.peek_shared_decode_attention(*args, **kw)
    torch.cuda.synchronize()
    others = [r for r in range(len(q)) if r not in (1, 2)]
    assert torch.equal(args[6][others], clean[others]) and torch.equal(args[6][2, 2:], clean[2, 2:])
    assert args[6][1].isnan().all()


def test_validation_on_request(monkeypatch):
    """Offsets, pages and lengths of rotation, reading and choice are looked at where that is asked for."""
    import paper_2607_02525_amd as P
    monkeypatch.setenv("PEEK_VALIDATE", "1")
    pool = P.KVPool(torch.zeros(4, 2, 1, 16, 64, dtype=torch.int8).cuda(), torch.ones(4, 2, 1).cuda())
    k = torch.zeros(20, 1, 64, dtype=BF).cuda()
    at, ctx = torch.tensor([0, 20]).cuda(), torch.zeros(1, dtype=I32).cuda()
    table = torch.tensor([[1, 2]], dtype=I32).cuda()
    freq = torch.ones(32, dtype=torch.float64).cuda()
    out = [torch.zeros_like(k) for _ in range(2)]

    def rotate(at=at, ctx=ctx, table=table, pool=pool):
        P.peek_rotate_append(None, k, None if pool is None else k, at, ctx, freq, None, k_out=out[0], pool=pool,
                             block_table=table if pool is not None else None)

    def read(at=at, ctx=ctx, table=table):
        P.peek_kv_read(pool, at, ctx, table, *out)

    rotate()
    rotate(pool=None)
    read()
    bounds = torch.zeros(4, 1, 2, 64, dtype=torch.int8).cuda()
    P.peek_kv_bounds(pool, None, torch.tensor([20], dtype=I32).cuda(), table, bounds)
    for call in (rotate, read):
        for kw in (dict(at=torch.tensor([0, 21]).cuda()), dict(at=torch.tensor([5, 4]).cuda()),
                   dict(table=torch.tensor([[1, 4]], dtype=I32).cuda()), dict(ctx=torch.tensor([13], dtype=I32).cuda())):
            with pytest.raises(P.PeekError) as e:
                call(**kw)
            assert e.value.status == P.PEEK_ERR_INVALID_ARGUMENT
    with pytest.raises(P.PeekError):
        rotate(at=torch.tensor([-1, 3]).cuda(), pool=None)
    with pytest.raises(P.PeekError):
        P.peek_kv_bounds(pool, None, torch.tensor([33], dtype=I32).cuda(), table, bounds)


@pytest.mark.parametrize("held", [0, 40])
@pytest.mark.parametrize("n,G,B", [(5, 4, 16), (40, 8, 16), (5, 2, 8)])
def test_a_first_member_without_tokens(held, n, G, B):
    """A padded row at a group's head: its pages stand for the others' shared keys, its own answer has none of them."""
    import paper_2607_02525_amd as P
    from tests.test_gpu_shared import grouped_pool
    gen = torch.Generator().manual_seed(held + n)
    codes, scales, table, contexts = grouped_pool(gen, [(128, [9, 5, 0, 70] + [3] * (n - 4))], B, 2, 64, F8)
    contexts = [held, *contexts[1:]]
    q = torch.randn(n, 2 * G, 64, generator=gen).to(BF)
    pool = P.KVPool(codes.cuda(), scales.cuda())
    out, lse = torch.full_like(q, math.nan).cuda(), torch.full((n, 2 * G), math.nan).cuda()
    ws = torch.empty(max(256, P.peek_shared_decode_attention_workspace(pool, n, 2 * G, table.shape[1], 1)),
                     dtype=torch.uint8).cuda()
    P.peek_shared_decode_attention(pool, q.cuda(), torch.tensor(contexts, dtype=I32).cuda(), table.cuda(),
                                   torch.tensor([0, n], dtype=I32).cuda(), torch.tensor([128], dtype=I32).cuda(), out,
                                   ws, lse=lse)
    for r, c in enumerate(contexts):
        if c == 0:
            assert out[r].abs().max() == 0 and (lse[r] == -math.inf).all()
            continue
        row = table[r].clone()
        if c >= 128:
            row[:128 // B] = table[0, :128 // B]
        k, v = R.cached(codes, scales, row, c)
        want, wl, _, spread, reach = R.attend(q[r:r + 1], k, v, 0.125, c)
        near(out[r:r + 1], want, R.out_bound(want, spread, reach, BF, c, R.most_of(scales, F8)), f"sequence {r}")
        near(lse[r:r + 1], wl, R.lse_bound(wl, reach, 64), f"lse of {r}")
