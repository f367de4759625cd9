"""GPU test of the example of shared prefixes and chosen blocks: what its last steps gave is attention in 64 bits over
what the cache holds."""
import importlib.util
import os
import sys

import numpy as np
import pytest

import peek_workloads as W
from tests import kv_reference as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
EXAMPLES = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples")


@pytest.mark.parametrize("workload,format", [("tiny", torch.float8_e4m3fn), ("rag", torch.int8)])
def test_the_example_generates(workload, format):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("decode_shared", os.path.join(EXAMPLES, "decode_shared.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    w = W.make("tiny", 42) if workload == "tiny" else W.make_rag(7, n=12, n_cached=128)
    keep, steps, H, G, D = 6, 3, 2, 4, 64
    r = example.generate(w, steps=steps, keep=keep, format=format)
    torch.cuda.synchronize()
    assert int(r["shared"].max()) > 0, "the queue shares nothing"
    pages, scales, table = r["pool"].pages.cpu(), r["pool"].scales.cpu(), r["table"].cpu()
    np.testing.assert_array_equal(r["dense"]["context"].cpu().numpy(), w.lengths + steps)
    # the pages have grown by `steps` tokens since, whose rows may have made a block's scale larger: only sequences whose
    # last block was begun after it are still what that step saw
    ctx, dense = r["context"].cpu().tolist(), r["dense"]
    seen = [i for i in range(w.n) if (w.lengths[i] + steps) % 16 == 0]
    for i in seen:
        k, v = R.cached(pages, scales, table[i], int(w.lengths[i]) + steps)
        check(dense["q"][i:i + 1].cpu(), k, v, dense["out"][i:i + 1], dense["lse"][i:i + 1], D)
    kept, tokens = r["kept"].cpu(), r["tokens_kept"].cpu()
    for i in range(w.n):
        nb = -(-ctx[i] // 16)
        for h in range(H):
            t = int(tokens[i, h])
            assert t == ctx[i] - 16 * max(0, nb - keep)
            rows = slice(h * G, (h + 1) * G)
            k, v = R.cached(pages[:, :, h:h + 1], scales[:, :, h:h + 1], kept[i, h], t)
            check(r["q"][i:i + 1, rows].cpu(), k, v, r["out"][i:i + 1, rows], r["lse"][i:i + 1, rows], D)
    k, v = R.cached(pages, scales, table[0], ctx[0])
    for got, want in zip(r["back"], (k, v)):
        assert torch.equal(got.cpu(), want.float().to(torch.bfloat16))


def check(q, k, v, out, lse, dim):
    want, wl, _, spread, reach = R.attend(q, k, v, dim ** -0.5, len(k))
    assert ((out.double().cpu() - want).abs() <= R.out_bound(want, spread, reach, torch.bfloat16)).all()
    assert ((lse.double().cpu() - wl).abs() <= R.lse_bound(wl, reach, dim)).all()
