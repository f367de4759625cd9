"""Host-only checks of arguments that the attention calls must not take at their word: the binding's and the entry
points' refusals beyond those of tests/test_attention_args.py. Fake device pointers are never read."""
import pytest

import paper_2607_02525_amd as P

torch = pytest.importorskip("torch")


def test_tables_whose_rows_overlap_are_refused():
    """A row expanded to all sequences, or rows closer than they are wide, have no stride that the calls take."""
    i32 = torch.int32
    row = torch.arange(6, dtype=i32)
    for t in (row[None].expand(3, -1), row.as_strided((3, 4), (1, 1)), row[None, :1].expand(4, -1)):
        with pytest.raises(ValueError, match="overlap"):
            P._table(t, t.shape[0])
    # rows of any stride from their width on get as far as the check for a device tensor, as do single and empty ones
    wide = torch.zeros(3, 9, dtype=i32)
    for t in (wide, wide[:, :4], wide[::2], wide[:1, :4], row[None].expand(1, -1), torch.zeros(3, 0, dtype=i32)):
        with pytest.raises(ValueError, match="device tensor"):
            P._table(t, t.shape[0])


def test_rows_of_another_shape_are_refused():
    """Enough elements are not enough: a weight per block of another width would be read and written at wrong places."""
    f32 = torch.float32
    for shape in ((3, 2, 9), (3, 2, 4), (3, 5, 2), (2, 2, 5), (6, 9), (3, 18), (3, 1, 2, 9), (2, 10)):
        with pytest.raises(ValueError, match="mass must be"):
            P._row_arg(torch.zeros(shape), "mass", f32, 3, 2, 5)
    with pytest.raises(ValueError, match="at least 30"):
        P._row_arg(torch.zeros(29), "mass", f32, 3, 2, 5)
    with pytest.raises(TypeError, match="mass must be"):
        P._row_arg(torch.zeros(3, 2, 5).double(), "mass", f32, 3, 2, 5)
    assert P._row_arg(None, "mass", f32, 3, 2, 5) is None
    # the shape itself, more rows of it (a buffer for a larger batch), and the same elements in other numbers of
    # dimensions get as far as the device check
    for t in (torch.zeros(3, 2, 5), torch.zeros(4, 2, 5), torch.zeros(30), torch.zeros(64), torch.zeros(6, 5),
              torch.zeros(3, 10), torch.zeros(5, 10), torch.zeros(3, 1, 2, 5)):
        with pytest.raises(ValueError, match="device tensor"):
            P._row_arg(t, "mass", f32, 3, 2, 5)


FAKE = 0x10000


def attend(call, out_strides, tokens, heads, dim):
    """What the entry point says to an output of this layout; the workspace is too small, so that nothing is run."""
    p = P._PoolStruct(FAKE, FAKE, 8, 1, 16, dim, P.PEEK_TYPE_I8)
    ref = P.ctypes.byref(p)
    if call == "decode":
        return P._lib.peek_decode_attention(ref, tokens, 0, heads, FAKE, heads * dim, dim, FAKE, FAKE, 1 << 20, 1 << 20,
                                            1.0, FAKE, *out_strides, None, None, None, FAKE, 0, None)
    return P._lib.peek_prefill_attention(ref, 1, tokens, 0, heads, 1, dim, FAKE, heads * dim, dim, FAKE, dim, 0, FAKE,
                                         dim, 0, FAKE, FAKE, FAKE, 1 << 20, 1 << 20, 1.0, FAKE, *out_strides, None, FAKE,
                                         0, None)


def test_outputs_whose_rows_overlap_are_refused():
    """Against a count of the elements that rows share; strides in units of 8 over heads of 64."""
    seen = set()
    for call in ("decode", "prefill"):
        for tokens, heads in ((1, 1), (1, 3), (3, 1), (2, 2), (3, 4), (5, 3)):
            for ts in (0, 8, 56, 64, 72, 128, 192, 200, 256, 320, 100 * 8):
                for hs in (0, 8, 64, 72, 104, 128, 136, 192, 256, 320, 960):
                    places = {t * ts + h * hs + i for t in range(tokens) for h in range(heads) for i in range(64)}
                    apart = len(places) == tokens * heads * 64
                    status = attend(call, (ts, hs), tokens, heads, 64)
                    seen.add(apart)
                    if apart:
                        assert status == P.PEEK_ERR_WORKSPACE_TOO_SMALL, (call, tokens, heads, ts, hs)
                    else:
                        assert status == P.PEEK_ERR_INVALID_ARGUMENT and "overlap" in P.peek_last_error()
    assert seen == {True, False}
    for strides in ((1 << 62, 64), (64, 1 << 62)):
        assert attend("decode", strides, 1 << 16, 1 << 16, 64) == P.PEEK_ERR_WORKSPACE_TOO_SMALL


def test_evictions_into_arrays_that_overlap_are_refused():
    """Every output against every other array, by its first and its last bytes."""
    n, heads, width, stride = 3, 2, 40000, 40010
    row = n * width * 4
    size = {"ctx": n * 4, "table": ((n - 1) * stride + width) * 4, "mass": row * heads, "keep": n * 4, "ctx_out": n * 4,
            "table_out": row, "mass_out": row * heads, "freed": row, "num": n * 4,
            "ws": P._lib.peek_kv_evict_workspace(n, heads, width)}
    far = {name: (i + 1) << 32 for i, name in enumerate(size)}

    def evict(at):
        status = P._lib.peek_kv_evict(n, heads, 16, at["ctx"], at["table"], width, stride, at["mass"], at["keep"], 0, 1,
                                      at["ctx_out"], at["table_out"], at["mass_out"], at["freed"], at["num"], at["ws"],
                                      size["ws"], None)
        return status, P.peek_last_error()

    outputs = ("ctx_out", "table_out", "mass_out", "freed", "num")
    for out in outputs:
        for other in size:
            if other == out:
                continue
            for at in (far[other], far[other] + size[other] - 4, far[other] - size[out] + 4):
                if (out, other, at) == ("ctx_out", "ctx", far["ctx"]):
                    continue
                status, message = evict({**far, out: at})
                assert status == P.PEEK_ERR_INVALID_ARGUMENT and "overlap" in message, (out, other)


def test_a_pool_keeps_its_tensors():
    """Other pages or scales cannot be put into a pool, whose calls would go on with the memory of the first."""
    for name in ("pages", "scales"):
        assert isinstance(getattr(P.KVPool, name), property) and getattr(P.KVPool, name).fset is None
