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


# --------------------------------------------------- infinities and NaN by place
@pytest.mark.parametrize("dtype,D", [(BF, 128), (HF, 64)])
@pytest.mark.parametrize("kind", ["cached", "parts", "many"])
def test_values_that_are_no_numbers_reach_the_rows_that_see_them(kind, dtype, D):
    """As over one uncached prompt: after a cached prefix (odd tiles are counted from another one), in keys split into
    parts (one of which has the odd value), and with more sequences than are counted."""
    gen = torch.Generator().manual_seed(16)
    H, G, B = 2, 3, 16
    held, new = {"cached": ([300, 64], [150, 70]), "parts": ([0], [2100]), "many": ([0, 16, 40] * 24, [33, 9, 70] * 24)}[kind]
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
