"""GPU test of the serving example on a queue whose prompts are all cached whole: nothing is left to prefill, and the
steps decode from shared pages alone."""
import importlib.util

import numpy as np
import pytest

import peek_workloads as W
from tests import kv_reference as R
from tests.test_gpu_serve_queue import PATH

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def test_a_queue_that_is_cached_whole():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("serve_queue", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    B, steps, keep = 16, 3, 24
    cached = [np.arange(1, 1 + 480, dtype=np.int32), np.arange(9, 9 + 64, dtype=np.int32)]
    prompts = [cached[0], cached[0][:64], cached[1], cached[0][:480], cached[1][:16]]
    pack = lambda xs: (np.concatenate(xs), np.cumsum([0] + [len(x) for x in xs]))
    w = W.Workload("cached", 0, *pack(prompts), block_size=B, threshold=32, cache_sequences=pack(cached))
    r = example.serve(w, steps=steps, keep=keep)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(r["h"], w.lengths)
    context = r["context"].cpu().numpy()
    gone = np.maximum(0, -(-(w.lengths + steps) // B) - keep)
    np.testing.assert_array_equal(context, w.lengths + 2 * steps - B * gone)
    pages, scales, table = r["pool"].pages.cpu(), r["pool"].scales.cpu(), r["table"].cpu().numpy()
    out, q = r["out"].double().cpu(), r["q"].cpu()
    for i in range(w.n):
        k, v = R.cached(pages, scales, table[i], int(context[i]))
        want, _, _, spread, reach = R.attend(q[i:i + 1], k, v, 64 ** -0.5, int(context[i]))
        assert ((out[i:i + 1] - want).abs() <= R.out_bound(want, spread, reach, torch.bfloat16)).all(), i
