"""GPU test of the serving example: the queue runs through match, prefill, decode and eviction, and the last step's
outputs are those of attention in 64 bits over what the cache then holds."""
import importlib.util
import os

import numpy as np
import pytest

import peek_workloads as W
from tests import kv_reference as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_queue.py")


@pytest.mark.parametrize("format", [torch.float8_e4m3fn, torch.int8])
def test_the_example_serves_a_queue(format):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("serve_queue", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    w, keep, steps, B = W.make("tiny", 42), 24, 5, 16
    r = example.serve(w, steps=steps, keep=keep, format=format)
    torch.cuda.synchronize()
    blocks = -(-(w.lengths + steps) // B)
    np.testing.assert_array_equal(r["freed"].cpu().numpy(), np.maximum(0, blocks - keep))
    context = r["context"].cpu().numpy()
    np.testing.assert_array_equal(context, w.lengths + 2 * steps - B * np.maximum(0, blocks - keep))
    pages, scales, table = r["pool"].pages.cpu(), r["pool"].scales.cpu(), r["table"].cpu().numpy()
    out, lse, q = r["out"].double().cpu(), r["lse"].double().cpu(), r["q"].cpu()
    for i in range(w.n):
        k, v = R.cached(pages, scales, table[i], int(context[i]))
        want, wl, _, spread, reach = R.attend(q[i:i + 1], k, v, 64 ** -0.5, int(context[i]))
        assert ((out[i:i + 1] - want).abs() <= R.out_bound(want, spread, reach, torch.bfloat16)).all(), i
        assert ((lse[i:i + 1] - wl).abs() <= R.lse_bound(wl, reach, 64)).all(), i
    # every token since the eviction put its weight somewhere: kv heads times their query heads, once a step
    weight = r["mass"].double().sum((1, 2)).cpu()
    assert (weight > 8 * steps * 0.99).all()
