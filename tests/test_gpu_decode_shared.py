"""GPU test of the example of shared prefixes and chosen blocks: what its last steps gave is attention in 64 bits over
what the cache holds."""
import importlib.util
import os
import sys

import numpy as np
import pytest

import peek_workloads as W
from tests import kv_reference as R
from tests import step_reference as S

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


@pytest.mark.parametrize("workload,format", [("tiny", torch.int8), ("rag", torch.float8_e4m3fn)])
def test_every_step_of_the_example(workload, format, monkeypatch):
    """All sequences of every shared step, over what the cache held then, and the blocks of every choice."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("decode_shared", os.path.join(EXAMPLES, "decode_shared.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    dense, choices = [], []
    attend, choose = example.peek_shared_decode_attention, example.peek_block_select

    def shared_step(pool, q, context, table, group_offsets, shared, out, ws, members, lse):
        attend(pool, q, context, table, group_offsets, shared, out, ws, members=members, lse=lse)
        at = [x.cpu() for x in (pool.pages, pool.scales, q, context, table, group_offsets, shared, members, out, lse)]
        dense.append([x.clone() for x in at])

    def choice(pool, bounds, q, context, table, sink, recent, tokens, kept, ws):
        choose(pool, bounds, q, context, table, sink, recent, tokens, kept, ws)
        at = [x.cpu().clone() for x in (pool.pages, pool.scales, bounds, q, context, table, tokens, kept)]
        choices.append(at + [sink, recent])

    monkeypatch.setattr(example, "peek_shared_decode_attention", shared_step)
    monkeypatch.setattr(example, "peek_block_select", choice)
    w = W.make("tiny", 42) if workload == "tiny" else W.make_rag(7, n=12, n_cached=128)
    steps, keep, H, G, D, B = 2, 6, 2, 4, 64, 16
    example.generate(w, steps=steps, keep=keep, format=format)
    assert len(dense) == len(choices) == steps
    for pages, scales, q, context, table, offsets, shared, members, out, lse in dense:
        sizes = offsets.diff().tolist()
        together = sum(m for m, s in zip(sizes, shared.tolist()) if s >= B and m > 1)
        assert together > 1, "no sequence shares anything"
        assert sorted(members.tolist()) == list(range(w.n))
        for r in range(w.n):
            t = int(context[r])
            k, v = R.cached(pages, scales, table[r], t)
            check(q[r:r + 1], k, v, out[r:r + 1], lse[r:r + 1], D)
    beyond = 0
    for pages, scales, bounds, q, context, table, tokens, kept, sink, recent in choices:
        for r in range(w.n):
            nb = -(-int(context[r]) // B)
            beyond += nb > keep
            ids = table[r, :nb].long()
            for p in {int(x) for x in ids[:-1]}:
                hi, lo = S.bounds(pages, scales, p, B)
                assert np.array_equal(bounds[p, :, 0].numpy(), hi) and np.array_equal(bounds[p, :, 1].numpy(), lo)
            for h in range(H):
                x = bounds[ids, h].numpy().astype(np.int64)
                score = S.scores(q[r, h * G:(h + 1) * G], x[:, 0], x[:, 1], scales[ids, 0, h].numpy(), format)
                stay = S.choose(score, nb, keep, sink, recent)
                assert kept[r, h].tolist() == table[r, stay].tolist() + [-1] * (keep - len(stay))
                assert int(tokens[r, h]) == int(context[r]) - B * (nb - len(stay))
    assert beyond > 0, "nothing was left out of a choice"
