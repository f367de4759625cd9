"""GPU tests of attention over sequences as long as a table can name, close to 2^31 tokens: every block but the last is
one page, so that the sums over all of it are known."""
import math

import pytest

from tests import kv_reference as R
from tests.test_gpu_attention import BF, F8, I8, JUNK, near

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("B,fmt,tokens", [(256, I8, 2 ** 31 - 256), (256, I8, 2 ** 31 - 256 - 100),
                                          (4, F8, 2 ** 31 - 5), (16, F8, 2 ** 31 - 16 - 3)])
def test_lengths_close_to_the_end_of_32_bits(B, fmt, tokens):
    import paper_2607_02525_amd as P
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    D, W = 64, (2 ** 31 - 1) // B
    last, live = (tokens - 1) // B, (tokens - 1) % B + 1
    codes = torch.zeros(2, 2, 1, B, D)
    codes[0, 1] = 3
    codes[1, 0, 0, :, 0] = 40
    codes[1, 1, 0] = (torch.arange(B) % 8 + 1)[:, None].float()
    codes = codes.to(fmt)
    codes.view(torch.uint8)[1, :, :, live:] = JUNK[fmt]
    pool = P.KVPool(codes.cuda(), torch.ones(2, 2, 1).cuda())
    table = torch.zeros(1, W, dtype=torch.int32, device="cuda")
    table[0, last] = 1
    held = torch.tensor([tokens], dtype=torch.int32).cuda()
    q = torch.zeros(1, 2, D, dtype=BF)
    q[0, 0, 0] = 1                        # this head looks at the last block, the other at all tokens alike
    dq, own = q.cuda(), torch.zeros(1, 1, D, dtype=BF).cuda()
    mean = (torch.arange(live) % 8 + 1).double().mean()
    many, few = tokens - live, live * math.exp(40)
    out, lse, with_mass = torch.empty_like(dq), torch.empty(1, 2).cuda(), B == 256
    mass = torch.empty(1, 1, W).cuda() if with_mass else None
    ws = torch.empty(max(256, P.peek_decode_attention_workspace(pool, 1, 2, W, mass=with_mass)), dtype=torch.uint8).cuda()
    P.peek_decode_attention(pool, dq, held, table, out, ws, scale=1.0, lse=lse, mass=mass)
    torch.cuda.synchronize()

    def check(extra, what):               # `extra` tokens of logit 0 and no value
        sums = torch.tensor([many + few + extra, tokens + extra]).double()
        value = torch.tensor([3 * many + few * mean, 3 * many + live * mean]).double() / sums
        near(out, value[None, :, None].expand(1, 2, D), 2.0 ** -7 * value[None, :, None], what)
        near(lse, sums.log()[None], R.lse_bound(sums.log()[None], 40.0, D), f"{what}'s lse")

    check(0, "decode")
    if with_mass:
        share = torch.tensor([few / (many + few) + live / tokens, 1 / (many + few) * B + B / tokens]).double()
        near(mass[0, 0, [last, 0]], share, 2.0 ** -12 * share, "mass")
        rest = mass[0, 0, 1:last]
        assert rest.min() == rest.max() and (last + 1 == W or mass[0, 0, last + 1:].abs().max() == 0)
    del ws, mass
    ws = torch.empty(max(256, P.peek_prefill_attention_workspace(1, 1, 2, 1, D, W * B)), dtype=torch.uint8).cuda()
    P.peek_prefill_attention(dq, own, own, torch.tensor([0, 1]).cuda(), out, ws, pool=pool, prefix=held,
                             block_table=table, scale=1.0, lse=lse)
    torch.cuda.synchronize()
    check(1, "prefill")
