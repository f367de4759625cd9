"""GPU tests of attention at the ends of its ranges: weights that differ by many orders of magnitude, scales of zero
and at their limits, logits of any size, infinities after a cached prefix, lengths and page ids that the table does not
have. The other side is tests/kv_reference.py's sums in 64 bits."""
import math

import pytest

from tests import kv_reference as R
from tests.test_gpu_attention import BF, F8, HF, I8, make_pool, near

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def decode(q, codes, scales, table, contexts, scale, with_mass=False):
    import paper_2607_02525_amd as P
    n, Hq, _ = q.shape
    H, W = codes.shape[2], table.shape[1]
    pool, dq = P.KVPool(codes.cuda(), scales.cuda()), q.cuda()
    out, lse = torch.empty_like(dq), torch.full((n, Hq), math.nan).cuda()
    mass = torch.full((n, H, W), math.nan).cuda() if with_mass else None
    ws = torch.full((max(256, P.peek_decode_attention_workspace(pool, n, Hq, W, mass=with_mass)),), 0xFF,
                    dtype=torch.uint8).cuda()
    P.peek_decode_attention(pool, dq, torch.tensor(contexts, dtype=torch.int32).cuda(), table.cuda(), out, ws,
                            scale=scale, lse=lse, mass=mass)
    torch.cuda.synchronize()
    return (out, lse, mass) if with_mass else (out, lse)


def prefill(q, k, v, new, scale, codes=None, scales=None, table=None, held=None):
    """new, held: own and cached tokens of every sequence."""
    import paper_2607_02525_amd as P
    T, Hq, D = q.shape
    dq, more, width = q.cuda(), {}, 0
    if codes is not None:
        width = table.shape[1] * codes.shape[3]
        more = dict(pool=P.KVPool(codes.cuda(), scales.cuda()), prefix=torch.tensor(held, dtype=torch.int32).cuda(),
                    block_table=table.cuda())
    offsets = torch.tensor([0] + torch.tensor(new).cumsum(0).tolist()).cuda()
    out, lse = torch.empty_like(dq), torch.full((T, Hq), math.nan).cuda()
    ws = torch.full((max(256, P.peek_prefill_attention_workspace(len(new), T, Hq, k.shape[1], D, width)),), 0xFF,
                    dtype=torch.uint8).cuda()
    P.peek_prefill_attention(dq, k.cuda(), v.cuda(), offsets, out, ws, scale=scale, lse=lse, **more)
    torch.cuda.synchronize()
    return out, lse


# ------------------------------------------- many small weights beside a large one
def faint_bound(out, spread, reach, dtype, weights, values, scales):
    """As kv_reference's out_bound, but what is lost of a weight below the type's normal range is held against the
    64 keys around it, not against the row: a weight times its value's scale is off by at most 2^-17 of the largest such
    product there. weights [T, S] of one head, values [S, D], scales [S] of the values."""
    S = scales.numel()
    u, delta = R.ROUNDOFF[dtype], R.logit_error(reach, out.shape[-1])[..., None]
    product = torch.nn.functional.pad(weights * scales, (0, -S % 64)).view(weights.shape[0], -1, 64).amax(2)
    codes = torch.nn.functional.pad((values / scales[:, None]).abs(), (0, 0, 0, -S % 64)).view(-1, 64, values.shape[1])
    lost = 2.0 ** -17 * (product @ codes.sum(1))
    return u * out.abs() + (1 + u) * (u + 2.1 * delta + 2.0 ** -18) * spread + lost[:, None] + R.SMALLEST[dtype]


def faint_cache(gen, tokens, fmt, nats, ratio, B=16, D=128):
    """One token of a large logit (nats above all others) and no value, in a first block whose V scale is `ratio` times
    the others'; 63 more tokens without a value; and `tokens` in all."""
    blocks = -(-tokens // B)
    codes = torch.zeros(blocks, 2, 1, B, D)
    codes[0, 0, 0, 0, 0] = nats
    codes[64 // B:, 1] = (torch.rand(blocks - 64 // B, 1, B, D, generator=gen) * 60).round() + 60
    scales = torch.ones(blocks, 2, 1)
    scales[:, 1] = 1 / 64
    scales[0, 1] = ratio / 64
    codes = codes.to(F8) if fmt == F8 else codes.to(I8)
    return codes, scales, torch.arange(blocks, dtype=torch.int32)[None]


@pytest.mark.parametrize("fmt", [F8, I8])
@pytest.mark.parametrize("ratio", [1.0, 16.0, 64.0, 4096.0])
def test_faint_weights_of_f16_rows_over_a_cache(fmt, ratio):
    """24000 keys 14 nats below one without a value: together they have 2% of the weight, and are all of the output."""
    gen = torch.Generator().manual_seed(1)
    T, D = 24000, 128
    codes, scales, table = faint_cache(gen, T, fmt, 14.0, ratio)
    q = torch.zeros(3, 2, D, dtype=HF)
    q[..., 0] = 1
    keys, values = R.cached(codes, scales, table[0], T)
    per_key = scales[:, 1, 0].double().repeat_interleave(16)
    want, wl, w, spread, reach = R.attend(q[:1], keys, values, 1.0, T)
    bound = faint_bound(want, spread, reach, HF, w[0], values[:, 0], per_key)
    assert (bound < 2.0 ** -9 * want).all()
    out, lse = decode(q[:1], codes, scales, table, [T], 1.0)
    near(out, want, bound, "decode")
    near(lse, wl, R.lse_bound(wl, reach, D), "decode's lse")
    own = torch.zeros(3, 1, D, dtype=HF)
    out, lse = prefill(q, own, own, [3], 1.0, codes, scales, table, [T])
    for i in range(3):
        want, wl, w, spread, reach = R.attend(q[i:i + 1], torch.cat([keys, own[:i + 1].double()]),
                                              torch.cat([values, own[:i + 1].double()]), 1.0, T + i + 1)
        # (the own tokens' values are 0: they have a part in the sum of weights alone)
        bound = faint_bound(want, spread, reach, HF, w[0, :, :T], values[:, 0], per_key)
        near(out[i:i + 1], want, bound, f"prefill, row {i}")
        near(lse[i:i + 1], wl, R.lse_bound(wl, reach, D), f"prefill's lse, row {i}")


@pytest.mark.parametrize("nats", [10.0, 14.0, 16.0])
def test_faint_weights_of_f16_rows_over_own_tokens(nats):
    gen = torch.Generator().manual_seed(2)
    T, D = 12000, 64
    q, k, v = torch.zeros(T, 1, D, dtype=HF), torch.zeros(T, 1, D, dtype=HF), torch.zeros(T, 1, D, dtype=HF)
    q[..., 0] = 1
    k[0, 0, 0] = nats
    v[64:] = (torch.rand(T - 64, 1, D, generator=gen) + 1).to(HF)
    out, lse = prefill(q, k, v, [T], 1.0)
    for i in (100, 1023, 5000, T - 1):
        want, wl, w, spread, reach = R.attend(q[i:i + 1], k[:i + 1], v[:i + 1], 1.0, i + 1)
        bound = faint_bound(want, spread, reach, HF, w[0], v[:i + 1, 0].double(), torch.ones(i + 1).double())
        near(out[i:i + 1], want, bound, f"row {i}")
        near(lse[i:i + 1], wl, R.lse_bound(wl, reach, D), f"lse of row {i}")


def test_faint_weights_between_large_ones():
    """Tiles of large and of small V scales by turns, 2^14 apart, and logits that lie far apart too: what a row has
    summed is brought to the size of the tile at hand and back."""
    gen = torch.Generator().manual_seed(3)
    T, D, B = 3000, 128, 16
    for fmt in (F8, I8):
        codes, scales, table = make_pool(gen, [T], 1, B, D, fmt, spread=1)
        turn = torch.arange(T).div(B, rounding_mode="floor") // 4 % 2
        for b in range(table.shape[1]):
            scales[table[0, b].long(), 1] *= 2.0 ** (-12 if turn[b * B] else 2)
        for q_spread in (1.0, 12.0):
            q = (torch.randn(1, 4, D, generator=gen) * q_spread).to(HF)
            keys, values = R.cached(codes, scales, table[0], T)
            s = D ** -0.5
            want, wl, w, spread, reach = R.attend(q, keys, values, s, T)
            per_key = scales[table[0].long(), 1, 0].double().repeat_interleave(B)[:T]
            bound = torch.cat([faint_bound(want[:, h:h + 1], spread[:, h:h + 1], reach[:, h:h + 1], HF, w[h],
                                           values[:, 0], per_key) for h in range(4)], 1)
            out, lse, mass = decode(q, codes, scales, table, [T], s, with_mass=True)
            near(out, want, bound, "decode")
            near(lse, wl, R.lse_bound(wl, reach, D), "decode's lse")
            share = torch.zeros(table.shape[1] * B, dtype=torch.float64)
            share[:T] = w[:, 0].sum(0)
            share = share.view(-1, B).sum(1)
            near(mass[0, 0], share, R.mass_bound(share, reach.amax(), share), "mass")
            own = torch.zeros(1, 1, D, dtype=HF)
            out, lse = prefill(q, own, own, [1], s, codes, scales, table, [T])
            want, wl, w, spread, reach = R.attend(q, torch.cat([keys, own.double()]),
                                                  torch.cat([values, own.double()]), s, T + 1)
            bound = torch.cat([faint_bound(want[:, h:h + 1], spread[:, h:h + 1], reach[:, h:h + 1], HF, w[h][:, :T],
                                           values[:, 0], per_key) for h in range(4)], 1)
            near(out, want, bound, "prefill")
            near(lse, wl, R.lse_bound(wl, reach, D), "prefill's lse")


# ------------------------------------------------------------------- scales
SCALED = [(BF, F8, 16, 128), (BF, I8, 16, 64), (HF, F8, 4, 64), (HF, I8, 8, 128), (HF, F8, 64, 128)]


@pytest.mark.parametrize("which", ["k", "v", "both"])
@pytest.mark.parametrize("dtype,fmt,B,D", SCALED)
def test_blocks_of_scale_zero(dtype, fmt, B, D, which):
    """Keys of scale 0 are 0, and so are values but for the 2^-60 that stands for a smaller scale: other blocks and the
    sums of weights stay right, in tiles that a sequence ends in too."""
    gen = torch.Generator().manual_seed(4)
    contexts, H, G = [1, 5, 63, 64, 100, 333, 700], 2, 3
    codes, scales, table = make_pool(gen, contexts, H, B, D, fmt)
    live = ~scales.isnan()
    zero = live & (torch.rand(scales.shape, generator=gen) < 0.4)
    if which != "both":
        zero[:, 1 if which == "k" else 0] = False
    scales[zero] = 0
    if which != "k":
        scales[table[0, 0].long(), 1] = 0                   # a sequence of nothing else
    check(gen, contexts, H, G, codes, scales, table, dtype, D, D ** -0.5)


def check(gen, contexts, H, G, codes, scales, table, dtype, D, scale, q_spread=1.0, new=2):
    n, W, B = len(contexts), table.shape[1], codes.shape[3]
    fmt, most = codes.dtype, R.most_of(scales, codes.dtype)
    q = (torch.randn(n, H * G, D, generator=gen) * q_spread).to(dtype)
    out, lse, mass = decode(q, codes, scales, table, contexts, scale, with_mass=True)
    meant = scales.clone()
    meant[:, 1] = scales[:, 1].clamp(min=2.0 ** -60)
    kv = [R.cached(codes, meant, table[r], c) for r, c in enumerate(contexts)]
    for r, c in enumerate(contexts):
        want, wl, w, spread, reach = R.attend(q[r:r + 1], *kv[r], scale, c)
        near(out[r:r + 1], want, R.out_bound(want, spread, reach, dtype, c, most), f"decode of {c} tokens")
        near(lse[r:r + 1], wl, R.lse_bound(wl, reach, D), f"decode's lse of {c} tokens")
        share = torch.zeros(H * G, W * B, dtype=torch.float64)
        share[:, :c] = w[:, 0]
        share = share.view(H, G, W, B).sum((1, 3))
        near(mass[r], share, R.mass_bound(share, reach.view(H, G).amax(1)[:, None], share), f"mass of {c} tokens")
    rows = (torch.randn(n * new, H * G, D, generator=gen) * q_spread).to(dtype)
    k, v = (torch.randn(n * new, H, D, generator=gen).to(dtype) for _ in range(2))
    out, lse = prefill(rows, k, v, [new] * n, scale, codes, scales, table, contexts)
    for r, c in enumerate(contexts):
        a, b = r * new, (r + 1) * new
        want, wl, _, spread, reach = R.attend(rows[a:b], torch.cat([kv[r][0], k[a:b].double()]),
                                              torch.cat([kv[r][1], v[a:b].double()]), scale, c + 1)
        near(out[a:b], want, R.out_bound(want, spread, reach, dtype, c + new, most), f"prefill after {c} tokens")
        near(lse[a:b], wl, R.lse_bound(wl, reach, D), f"prefill's lse after {c} tokens")


@pytest.mark.parametrize("fmt", [F8, I8])
@pytest.mark.parametrize("size", [2.0 ** -90, 2.0 ** -70, 2.0 ** 75])
def test_values_of_a_size_that_no_append_leaves(size, fmt):
    """A pool of another maker's, whose values are all that small or large, has its scales as they are."""
    gen = torch.Generator().manual_seed(10)
    contexts, H, G, D = [7, 90, 300], 2, 4, 64
    codes, scales, table = make_pool(gen, contexts, H, 16, D, fmt)
    scales[:, 1] *= size
    q = torch.randn(len(contexts), H * G, D, generator=gen).to(BF)
    out, lse = decode(q, codes, scales, table, contexts, D ** -0.5)
    k, v = torch.randn(3, H, D, generator=gen).to(BF), (torch.randn(3, H, D, generator=gen) * size).to(BF)
    pre, _ = prefill(q, k, v, [1] * 3, D ** -0.5, codes, scales, table, contexts)
    most = R.most_of(scales[:, 1], fmt) if size > 1 else 0.0
    for r, c in enumerate(contexts):
        keys, values = R.cached(codes, scales, table[r], c)
        want, wl, _, spread, reach = R.attend(q[r:r + 1], keys, values, D ** -0.5, c)
        near(out[r:r + 1], want, R.out_bound(want, spread, reach, BF, c, most), f"decode of {c} tokens")
        near(lse[r:r + 1], wl, R.lse_bound(wl, reach, D), f"decode's lse of {c} tokens")
        if size < 1:      # (an own value counts as of scale 1: beside it a cached one of 2^75 leaves nothing)
            want, wl, _, spread, reach = R.attend(q[r:r + 1], torch.cat([keys, k[r:r + 1].double()]),
                                                  torch.cat([values, v[r:r + 1].double()]), D ** -0.5, c + 1)
            near(pre[r:r + 1], want, R.out_bound(want, spread, reach, BF, c + 1, most), f"prefill after {c} tokens")


@pytest.mark.parametrize("fmt", [F8, I8])
def test_scales_at_their_limits(fmt):
    """The smallest and the largest scale that an append leaves (2^-60 of a block of zeros, 2^60), and a call's scale
    that takes a key's below the range of 32 bits."""
    gen = torch.Generator().manual_seed(5)
    contexts = [7, 90, 300]
    for k_scale, v_scale, scale in ((2.0 ** -60, 2.0 ** -60, 0.125), (2.0 ** -60, 0.01, 1e-30),
                                    (2.0 ** 40, 2.0 ** 60, 1e-14), (0.01, 2.0 ** 60, 0.125)):
        codes, scales, table = make_pool(gen, contexts, 2, 16, 64, fmt)
        live = ~scales.isnan()
        scales[:, 0] = torch.where(live[:, 0], k_scale, scales[:, 0])
        scales[:, 1] = torch.where(live[:, 1], v_scale, scales[:, 1])
        check(gen, contexts, 2, 4, codes, scales, table, BF, 64, scale)


def test_validation_reports_scales_out_of_range(monkeypatch):
    import paper_2607_02525_amd as P
    monkeypatch.setenv("PEEK_VALIDATE", "1")
    H, B, D = 2, 16, 64
    q, out = (torch.zeros(1, 2 * H, D, dtype=BF, device="cuda") for _ in range(2))
    k = torch.zeros(1, H, D, dtype=BF, device="cuda")
    one, table = torch.tensor([0, 1], device="cuda"), torch.tensor([[0, 2]], dtype=torch.int32, device="cuda")
    ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    # (K's, V's scale, where it is, the tokens held) and whether attention, and an append, may see it
    for part, x, page, held, seen, added in ((0, 0.0, 2, 20, True, True), (1, 0.0, 2, 20, True, True),
                                             (0, -1.0, 2, 20, True, False), (1, -1.0, 2, 20, False, False),
                                             (0, math.nan, 2, 20, False, False), (1, math.nan, 2, 20, False, False),
                                             (0, math.inf, 2, 20, False, False), (1, 2.0 ** 61, 2, 20, False, False),
                                             (1, math.nan, 0, 20, False, True), (1, math.nan, 2, 16, True, True),
                                             (1, math.nan, 1, 20, True, True)):
        scales = torch.ones(4, 2, H)
        scales[page, part, 1] = x
        pool = P.KVPool(torch.zeros(4, 2, H, B, D, dtype=torch.int8).cuda(), scales.cuda())
        ctx = torch.tensor([held], dtype=torch.int32).cuda()
        for right, call in ((seen, lambda: P.peek_decode_attention(pool, q, ctx, table, out, ws)),
                            (seen, lambda: P.peek_prefill_attention(q, k, k, one, out, ws, pool=pool, prefix=ctx,
                                                                    block_table=table)),
                            (added, lambda: P.peek_kv_append(pool, k, k, one, ctx, table))):
            if right:
                call()
                continue
            with pytest.raises(P.PeekError, match="scales") as e:
                call()
            assert e.value.status == P.PEEK_ERR_INVALID_ARGUMENT


# ------------------------------------------------------------------- logits
def steep(T, H, D, size, dtype, gen):
    """Keys whose logits are -size .. -2 size, each far from the next, the largest somewhere in the middle."""
    k = torch.zeros(T, H, D, dtype=dtype)
    order = torch.randperm(T, generator=gen)
    k[:, :, 0] = -(size * (1 + order.float() / T))[:, None].to(dtype)
    return k


SIZES = [3e7, 1e9, 1e12, 1e20, 1e29, 1e31, 1e36]


@pytest.mark.parametrize("dtype,size", [(HF, 3e7), (HF, 1e9), *((BF, x) for x in SIZES)])
def test_logits_of_any_size_over_own_tokens(dtype, size):
    """A row's sum of weights is at least that of its largest key, however large or far below 0 all of its logits are:
    the output is a value of the row's, or between several."""
    gen = torch.Generator().manual_seed(6)
    T, H, D = 200, 2, 64
    root = math.sqrt(size)
    k = steep(T, H, D, root, dtype, gen)
    v = (torch.rand(T, H, D, generator=gen) + 1).to(dtype)
    for sign in (1, -1):
        q = torch.zeros(T, H * 2, D, dtype=dtype)
        q[..., 0] = sign * root
        for new in ([T], [100, 0, 100]):
            out, lse = prefill(q, k, v, new, 1.0)
            a = 0
            for t in new:
                want, wl, w, _, reach = R.attend(q[a:a + t], k[a:a + t], v[a:a + t], 1.0, 1)
                want = want / w.sum(2).T[..., None]      # (64 bits too lose the logarithm of a sum beside 1e20)
                # a key's logit is the product of two numbers, rounded once, and times a power of two: keys that
                # differ in 8 bits stay in order, and equal ones share the weight
                near(out[a:a + t], want, 2.0 ** -7 * want.abs(), f"rows of {t} tokens")
                near(lse[a:a + t], wl, R.lse_bound(wl, reach, D), f"lse of {t} tokens")
                a += t


@pytest.mark.parametrize("dtype,fmt", [(BF, F8), (BF, I8), (HF, F8)])
@pytest.mark.parametrize("size", SIZES)
def test_logits_of_any_size_over_a_cache(size, dtype, fmt):
    gen = torch.Generator().manual_seed(7)
    B, D, contexts = 16, 64, [1, 50, 64, 300]
    codes, scales, table = make_pool(gen, contexts, 1, B, D, fmt)
    x = torch.zeros(codes.shape[0], 1, B, D)
    x[..., 0] = -96
    for r, c in enumerate(contexts):                         # one key above the others, one below
        for t, code in ((c // 2, -64), (c // 3, -120)):
            if c > 1:
                x[table[r, t // B].long(), 0, t % B, 0] = code
    ids = torch.cat([table[r, :-(-c // B)].long() for r, c in enumerate(contexts)])
    codes.view(torch.uint8)[ids, 0] = x.to(fmt).view(torch.uint8)[ids]
    root = 2.0 ** min(round(math.log2(size) / 2), 60)
    row = 2.0 ** round(math.log2(size / 64 / root)) if dtype == BF else 2.0 ** 10
    call = size / 64 / root / row if dtype == HF else 1.0
    scales[ids, 0] = root
    for sign in (1, -1):
        q = torch.zeros(len(contexts), 2, D, dtype=dtype)
        q[..., 0] = sign * row
        out, lse, mass = decode(q, codes, scales, table, contexts, call, with_mass=True)
        rows = torch.zeros(len(contexts), 2, D, dtype=dtype)
        rows[..., 0] = sign * row
        far = torch.zeros(len(contexts), 1, D, dtype=dtype)      # an own key below all cached ones (float16: at 0)
        if dtype == BF:
            far[..., 0] = -sign * 448.0 * root
        pre, pre_lse = prefill(rows, far, far, [1] * len(contexts), call, codes, scales, table, contexts)
        for r, c in enumerate(contexts):
            keys, values = R.cached(codes, scales, table[r], c)
            want, wl, w, spread, reach = R.attend(q[r:r + 1], keys, values, call, c)
            near(out[r:r + 1], want, 2.0 ** -7 * spread, f"decode of {c} tokens")
            near(lse[r:r + 1], wl, R.lse_bound(wl, reach, D), f"decode's lse of {c} tokens")
            near(mass[r].sum(), torch.tensor(2.0).double(), torch.tensor(1e-4).double(), f"mass of {c} tokens")
            want, wl, w, spread, reach = R.attend(rows[r:r + 1], torch.cat([keys, far[r:r + 1].double()]),
                                                  torch.cat([values, far[r:r + 1].double()]), call, c + 1)
            near(pre[r:r + 1], want, 2.0 ** -7 * spread, f"prefill after {c} tokens")
            near(pre_lse[r:r + 1], wl, R.lse_bound(wl, reach, D), f"prefill's lse after {c} tokens")


# --------------------------------------------------- infinities and NaN by place
@pytest.mark.parametrize("dtype,D", [(BF, 128), (HF, 64)])
@pytest.mark.parametrize("kind", ["cached", "parts", "many"])
def test_values_that_are_no_numbers_reach_the_rows_that_see_them(kind, dtype, D):
    """As over one uncached prompt: after a cached prefix (odd tiles are counted from another one), in keys split into
    parts (one of which has the odd value), and with more sequences than are counted."""
    gen = torch.Generator().manual_seed(16)
    H, G, B = 2, 3, 16
    held, new = {"cached": ([300, 64], [150, 70]), "parts": ([0], [2100]),
                 "many": ([0, 16, 40] * 24, [33, 9, 70] * 24)}[kind]
    T, at = sum(new), [0]
    for x in new:
        at.append(at[-1] + x)
    codes, scales, table = make_pool(gen, held, H, B, D, F8)
    q, k, v = ((torch.randn(T, h, D, generator=gen)).to(dtype) for h in (H * G, H, H))
    for r in range(0, len(new), 5):
        a, t = at[r], new[r]
        v[a + t // 2, 0, 3], v[a + t - 2, 0, 4], v[a + t // 3, 1, 5] = math.nan, math.inf, -math.inf
        v[a + t - 1, 1], k[a + 2 * t // 3, 1, 1] = math.nan, math.nan
    out, lse = prefill(q, k, v, new, D ** -0.5, codes, scales, table, held)
    for r in range(len(new)):
        if kind == "many" and r % 5 and r > 20:
            continue
        a, b = at[r], at[r + 1]
        pk, pv = R.cached(codes, scales, table[r], held[r])
        for i in range(a, b) if kind != "parts" else (*range(a, b, 97), *range(b - 70, b)):
            want, wl, _, spread, reach = R.attend(q[i:i + 1], torch.cat([pk, k[a:i + 1].double()]),
                                                  torch.cat([pv, v[a:i + 1].double()]), D ** -0.5, held[r] + i - a + 1)
            most = R.most_of(scales, F8)
            bound = R.out_bound(want, spread, reach, dtype, held[r] + i - a + 1, most).nan_to_num(0, 0)
            near(out[i:i + 1], want, bound, f"out of row {i - a} of sequence {r}")
            near(lse[i:i + 1], wl, R.lse_bound(wl, reach, D).nan_to_num(0, 0), f"lse of row {i - a} of sequence {r}")


# ------------------------------------------- lengths and page ids out of range
@pytest.mark.parametrize("B", [4, 16])
def test_lengths_and_pages_that_there_are_not(B):
    """Lengths are cut to 0 .. the table's tokens; a page outside the pool is page 0."""
    gen = torch.Generator().manual_seed(17)
    H, G, D, W = 2, 3, 64, 6
    codes, scales, table = make_pool(gen, [W * B] * 5, H, B, D, F8, spare=0)
    told = [-1, W * B + 1, 2 ** 31 - 1, W * B - 3, -2 ** 31]
    held = [0, W * B, W * B, W * B - 3, 0]
    wrong = table.clone()
    wrong[1, 2], wrong[3, 0], wrong[3, 5], wrong[2, 1] = -1, codes.shape[0], 2 ** 31 - 1, -2 ** 31
    for r, b in ((1, 2), (3, 0), (3, 5), (2, 1)):
        table[r, b] = 0
    q = torch.randn(5, H * G, D, generator=gen).to(BF)
    out, lse, mass = decode(q, codes, scales, wrong, told, D ** -0.5, with_mass=True)
    k, v = (torch.randn(5, H, D, generator=gen).to(BF) for _ in range(2))
    pre, pre_lse = prefill(q, k, v, [1] * 5, D ** -0.5, codes, scales, wrong, told)
    most = R.most_of(scales, F8)
    for r, c in enumerate(held):
        keys, values = R.cached(codes, scales, table[r], c) if c else (torch.zeros(0, H, D),) * 2
        want, wl, w, spread, reach = R.attend(q[r:r + 1], keys, values, D ** -0.5, c)
        near(out[r:r + 1], want, R.out_bound(want, spread, reach, BF, c, most), f"decode of sequence {r}")
        near(lse[r:r + 1], wl, R.lse_bound(wl, reach, D), f"decode's lse of sequence {r}")
        share = torch.zeros(H * G, W * B, dtype=torch.float64)
        share[:, :c] = w[:, 0]
        share = share.view(H, G, W, B).sum((1, 3))
        near(mass[r], share, R.mass_bound(share, reach.view(H, G).amax(1)[:, None], share), f"mass of sequence {r}")
        want, wl, _, spread, reach = R.attend(q[r:r + 1], torch.cat([keys, k[r:r + 1].double()]),
                                              torch.cat([values, v[r:r + 1].double()]), D ** -0.5, c + 1)
        near(pre[r:r + 1], want, R.out_bound(want, spread, reach, BF, c + 1, most), f"prefill of sequence {r}")
        near(pre_lse[r:r + 1], wl, R.lse_bound(wl, reach, D), f"prefill's lse of sequence {r}")


# ------------------------------------------------------------ what else is refused
def test_outputs_of_other_shapes_are_refused():
    """Masses of a wider table than the call's, which a view of its leading columns makes easy, and the like."""
    import paper_2607_02525_amd as P
    H, B, D, n, W = 2, 16, 64, 3, 4
    f32, i32 = dict(dtype=torch.float32, device="cuda"), dict(dtype=torch.int32, device="cuda")
    pool = P.KVPool(torch.zeros(W, 2, H, B, D, dtype=torch.int8).cuda(), torch.ones(W, 2, H).cuda())
    q = torch.zeros(n, 2 * H, D, dtype=BF).cuda()
    k, out = torch.zeros(n, H, D, dtype=BF).cuda(), torch.empty_like(q)
    ctx, offsets = torch.full((n,), 40, **i32), torch.arange(n + 1).cuda()
    wide = torch.arange(W, **i32).repeat(n, 2)
    table, ws = wide[:, :W], torch.empty(1 << 16, dtype=torch.uint8).cuda()
    good, bad = torch.zeros(n, H, W, **f32), torch.zeros(n, H, 2 * W, **f32)
    P.peek_decode_attention(pool, q, ctx, table, out, ws, mass=good, mass_in=good, lse=torch.empty(n, 2 * H, **f32))
    for kw in (dict(mass=bad), dict(mass=good, mass_in=bad), dict(lse=torch.empty(2 * H, n, **f32))):
        with pytest.raises(ValueError, match="must be"):
            P.peek_decode_attention(pool, q, ctx, table, out, ws, **kw)
    with pytest.raises(ValueError, match="lse must be"):
        P.peek_prefill_attention(q, k, k, offsets, out, ws, lse=torch.empty(2 * H, n, **f32))
    keep, count, held = torch.full((n,), 2, **i32), torch.empty(n, **i32), torch.empty(n, **i32)
    outs = [torch.empty(n, W, **i32), torch.empty(n, H, W, **f32), torch.empty(n, W, **i32)]
    P.peek_kv_evict(ctx, table, good, keep, B, 0, 1, held, *outs, count, ws)
    for i, name in enumerate(("block_table_out", "mass_out", "freed")):
        other = list(outs)
        other[i] = torch.empty(*outs[i].shape[:-1], 2 * W, dtype=outs[i].dtype, device="cuda")
        with pytest.raises(ValueError, match=f"{name} must be"):
            P.peek_kv_evict(ctx, table, good, keep, B, 0, 1, held, *other, count, ws)
    torch.cuda.synchronize()


@pytest.mark.parametrize("W", [6, 9000])
def test_eviction_of_lengths_that_there_are_not(W):
    """Lengths are cut to 0 .. the table's tokens before blocks are counted, and so is the context that is left."""
    import paper_2607_02525_amd as P
    B, H, n = 16, 2, 5
    told = [-1, W * B + 1, 2 ** 31 - 1, W * B - 3, -2 ** 31]
    held = [0, W * B, W * B, W * B - 3, 0]
    i32 = dict(dtype=torch.int32, device="cuda")
    table = torch.arange(n * W, **i32).view(n, W)
    mass = torch.rand(n, H, W, device="cuda")
    keep, res = torch.full((n,), 4, **i32), []
    for lengths in (told, held):
        ctx, count = torch.tensor(lengths, **i32), torch.empty(n, **i32)
        outs = [torch.empty(n, W, **i32), torch.empty(n, H, W, device="cuda"), torch.empty(n, W, **i32)]
        ws = torch.empty(max(256, P.peek_kv_evict_workspace(n, H, W)), dtype=torch.uint8, device="cuda")
        P.peek_kv_evict(ctx, table, mass, keep, B, 1, 2, ctx, *outs, count, ws)
        torch.cuda.synchronize()
        res.append([ctx, *outs, count])
    assert all(torch.equal(a, b) for a, b in zip(*res))
    assert res[0][0].tolist() == [0, 4 * B, 4 * B, 4 * B - 3, 0]


def test_a_pool_keeps_its_tensors():
    """Other pages or scales cannot be put into a pool, whose calls would go on with the memory of the first."""
    import paper_2607_02525_amd as P
    pool = P.KVPool.empty(2, 1, 16, 64)
    pages, scales = pool.pages, pool.scales
    with pytest.raises(AttributeError):
        pool.pages = pages.clone()
    with pytest.raises(AttributeError):
        pool.scales = scales.clone()
    assert pool.pages is pages and pool.scales is scales and pool._struct.d_pages == pages.data_ptr()


@pytest.mark.parametrize("scale", [2.0 ** -105, -1e-33, 2.0 ** -120])
def test_scales_that_bring_large_products_down(scale):
    """bfloat16 rows of a size that only a very small scale brings to logits of a few."""
    gen = torch.Generator().manual_seed(8)
    H, G, D, contexts = 2, 3, 64, [1, 40, 130]
    codes, scales, table = make_pool(gen, contexts, H, 16, D, F8)
    size = 2.0 ** round(-math.log2(abs(scale)) / 2)
    scales[:, 0] *= size
    n, new = len(contexts), 50
    q = (torch.randn(n, H * G, D, generator=gen) * size / 8).to(BF)
    out, lse = decode(q, codes, scales, table, contexts, scale)
    rows = (torch.randn(n * new, H * G, D, generator=gen) * size / 8).to(BF)
    k, v = ((torch.randn(n * new, H, D, generator=gen) * x).to(BF) for x in (size, 1.0))
    pre, pre_lse = prefill(rows, k, v, [new] * n, scale, codes, scales, table, contexts)
    most = R.most_of(scales[:, 1], F8)
    for r, c in enumerate(contexts):
        keys, values = R.cached(codes, scales, table[r], c)
        want, wl, _, spread, reach = R.attend(q[r:r + 1], keys, values, scale, c)
        near(out[r:r + 1], want, R.out_bound(want, spread, reach, BF, c, most), f"decode of {c} tokens")
        near(lse[r:r + 1], wl, R.lse_bound(wl, reach, D), f"decode's lse of {c} tokens")
        a, b = r * new, (r + 1) * new
        want, wl, _, spread, reach = R.attend(rows[a:b], torch.cat([keys, k[a:b].double()]),
                                              torch.cat([values, v[a:b].double()]), scale, c + 1)
        near(pre[a:b], want, R.out_bound(want, spread, reach, BF, c + new, most), f"prefill after {c} tokens")
        near(pre_lse[a:b], wl, R.lse_bound(wl, reach, D), f"prefill's lse after {c} tokens")


@pytest.mark.parametrize("fmt", [F8, I8])
def test_lse_of_float16_rows_of_few_tokens(fmt):
    """Many rows whose lse is near 0, where an error of the logarithm's parts shows."""
    gen = torch.Generator().manual_seed(9)
    H, G, D, contexts = 4, 8, 64, [1 + i % 40 for i in range(300)]
    codes, scales, table = make_pool(gen, contexts, H, 16, D, fmt)
    q = torch.randn(len(contexts), H * G, D, generator=gen).to(HF)
    out, lse = decode(q, codes, scales, table, contexts, 1e-3)
    k, v = (torch.randn(len(contexts), H, D, generator=gen).to(HF) for _ in range(2))
    _, pre_lse = prefill(q, k, v, [1] * len(contexts), 1e-3, codes, scales, table, contexts)
    for r, c in enumerate(contexts):
        keys, values = R.cached(codes, scales, table[r], c)
        _, wl, _, _, reach = R.attend(q[r:r + 1], keys, values, 1e-3, c)
        near(lse[r:r + 1], wl, R.lse_bound(wl, reach, D), f"decode's lse of {c} tokens")
        _, wl, _, _, reach = R.attend(q[r:r + 1], torch.cat([keys, k[r:r + 1].double()]),
                                      torch.cat([values, v[r:r + 1].double()]), 1e-3, c + 1)
        near(pre_lse[r:r + 1], wl, R.lse_bound(wl, reach, D), f"prefill's lse after {c} tokens")


def test_small_weights_of_f16_rows_beside_a_middling_one():
    """Tiles whose largest weight is 2^-14 of the row's, and has no value, while the others are 2^-22 of it: below
    float16's normal numbers, and all of the output."""
    D, T = 64, 64 * 40
    logit = torch.full((T,), -15.25)
    logit[0], logit[64::64] = 0.0, -9.75
    value = torch.ones(T)
    value[:64], value[64::64] = 0.0, 0.0
    q = torch.zeros(64, 1, D, dtype=HF)
    q[..., 0] = 1
    k, v = torch.zeros(T + 64, 1, D, dtype=HF), torch.zeros(T + 64, 1, D, dtype=HF)
    k[:T, 0, 0], v[:T] = logit, value[:, None, None].to(HF)
    keys, values, one = k[:T].double(), v[:T].double(), torch.ones(T).double()
    want, wl, w, spread, reach = R.attend(q[:1], keys, values, 1.0, T)
    bound = faint_bound(want, spread, reach, HF, w[0], values[:, 0], one)
    rows = torch.zeros(T, 1, D, dtype=HF)
    rows[..., 0] = 1
    out, lse = prefill(rows, k[:T], v[:T], [T], 1.0)
    near(out[-1:], want, bound, "own tokens")
    near(lse[-1:], wl, R.lse_bound(wl, reach, D), "own tokens' lse")
    for B in (4, 16):
        codes = torch.zeros(T // B, 2, 1, B, D)
        codes[:, 0, 0, :, 0], codes[:, 1, 0] = (logit * 8).view(-1, B), value.view(-1, B, 1)
        scales = torch.ones(T // B, 2, 1)
        scales[:, 0] = 0.125
        table = torch.arange(T // B, dtype=torch.int32)[None]
        out, lse = decode(q[:1], codes.to(I8), scales, table, [T], 1.0)
        near(out, want, bound, "decode")
        near(lse, wl, R.lse_bound(wl, reach, D), "decode's lse")
        own = torch.zeros(64, 1, D, dtype=HF)
        own[..., 0] = -16
        out, lse = prefill(q, own, torch.zeros_like(own), [64], 1.0, codes.to(I8), scales, table, [T])
        near(out[:1] * float((1 + math.exp(-16 - wl[0, 0]))), want, bound, "cached tokens")
