"""GPU tests of appends to float8 blocks whose held scale is no power of two, as pools of other producers have them:
codes of every finite magnitude that leaves the scale as it is, against the quotient's definition (tests/kv_reference.py).
Many of these quotients are ties between two codes, which a product with the scale's reciprocal misses."""
import math

import pytest

from tests import kv_reference as R
from tests.test_gpu_attention import BF, F8, HF, near

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
H, D = 2, 128


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def magnitudes(dtype, scale):
    """Every number of the type, from 0 on, whose own scale would not be larger."""
    x = torch.arange(0, 1 << 15, dtype=torch.int32).to(torch.int16).view(dtype)
    return x[x.float() <= 448 * 2.0 ** math.floor(math.log2(scale))]


def rows(dtype, scales, tokens):
    """K and V [tokens, H, D]: of each (K or V, head) the numbers of its scale, cut or repeated; every third negative."""
    out = torch.empty(2, tokens, H, D, dtype=dtype)
    for part in range(2):
        for h in range(H):
            x = magnitudes(dtype, scales[part][h])
            x = x[torch.arange(tokens * D) % len(x)].clone()
            x[::3] = -x[::3]
            out[part, :, h] = x.view(tokens, D)
    return out[0], out[1]


SCALES = [((7.0, 7 / 64), (13 / 64, 7 / 128)), ((5.3 / 448, 1.1), (0.3, 13 / 1024)), ((4.0, 0.875), (7 * 2.0 ** -20, 13.0))]
KINDS = [(16, 9), (32, 31), (64, 61), (256, 255)]       # block, new tokens: in registers, and taken again


@pytest.mark.parametrize("through", ["append", "rotation"])
@pytest.mark.parametrize("dtype", [BF, HF], ids=str)
@pytest.mark.parametrize("kind", KINDS, ids=str)
@pytest.mark.parametrize("scales", SCALES, ids=str)
def test_codes_of_a_held_scale(scales, kind, dtype, through):
    import paper_2607_02525_amd as P
    block, each = kind
    print("[gpu] held scales", scales, kind, dtype, through, flush=True)
    # as many blocks as the numbers fill, one sequence to each
    n = -(-(1 << 15) // (each * D))
    held = block - each
    k, v = rows(dtype, scales, n * each)
    gen = torch.Generator().manual_seed(block)
    codes = (torch.randn(n, 2, H, block, D, generator=gen) * 100).clamp(-448, 448).to(F8)
    own = torch.tensor(scales, dtype=torch.float32).expand(n, 2, H).contiguous()
    pool = P.KVPool(codes.cuda(), own.cuda())
    offsets, context, table = [each * i for i in range(n + 1)], [held] * n, [[i] for i in range(n)]
    at, ctx = torch.tensor(offsets).cuda(), torch.tensor(context, dtype=torch.int32).cuda()
    ids = torch.tensor(table, dtype=torch.int32).cuda()
    if through == "append":
        P.peek_kv_append(pool, k.cuda(), v.cuda(), at, ctx, ids)
    else:
        P.peek_rotate_append(None, k.cuda(), v.cuda(), at, ctx, None, None, pool=pool, block_table=ids)
    torch.cuda.synchronize()
    want, want_scales = codes.double().numpy(), own.double().numpy()
    R.append(want, want_scales, k.double().numpy(), v.double().numpy(), offsets, context, table, F8)
    assert torch.equal(pool.scales.cpu(), own), "the held scales stay"
    near(pool.pages.cpu().double(), torch.from_numpy(want), torch.zeros(()), "codes")
