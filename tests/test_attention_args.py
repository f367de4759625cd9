"""Host-only checks of the calls on the cache's contents: what they refuse, before any GPU work, and how much scratch
they ask for. Fake device pointers are never read."""
import ctypes

import pytest

import paper_2607_02525_amd as P

torch = pytest.importorskip("torch")
LIB = P._lib
FAKE = ctypes.c_void_p(0x10000)
ODD = ctypes.c_void_p(0x10008)
BAD = P.PEEK_ERR_INVALID_ARGUMENT


def pool(**kw):
    f = dict(d_pages=0x10000, d_scales=0x10000, num_pages=8, kv_heads=2, block_size=16, head_dim=128,
             type=P.PEEK_TYPE_F8E4M3)
    f.update(kw)
    return P._PoolStruct(*(f[k] for k, _ in P._PoolStruct._fields_))


BAD_POOLS = [dict(d_pages=None), dict(d_scales=None), dict(d_pages=0x10008), dict(num_pages=0), dict(num_pages=1 << 31),
             dict(kv_heads=0), dict(kv_heads=1025), dict(block_size=2), dict(block_size=12), dict(block_size=512),
             dict(head_dim=96), dict(head_dim=0), dict(type=P.PEEK_TYPE_BF16), dict(type=9)]


def append(p, n=2, tokens=3, type=0, k=FAKE, ks=(256, 128), v=FAKE, vs=(256, 128), off=FAKE, ctx=FAKE, table=FAKE,
           blocks=4, stride=4):
    return LIB.peek_kv_append(None if p is None else ctypes.byref(p), n, tokens, type, k, *ks, v, *vs, off, ctx, table,
                              blocks, stride, None)


def prefill(p, n=2, tokens=3, type=0, hq=4, h=2, d=128, q=FAKE, qs=(512, 128), k=FAKE, ks=(256, 128), v=FAKE,
            vs=(256, 128), off=FAKE, prefix=FAKE, table=FAKE, blocks=4, stride=4, scale=1.0, out=FAKE, os=(512, 128),
            ws=FAKE, size=1 << 40):
    return LIB.peek_prefill_attention(None if p is None else ctypes.byref(p), n, tokens, type, hq, h, d, q, *qs, k, *ks,
                                      v, *vs, off, prefix, table, blocks, stride, scale, out, *os, None, ws, size, None)


def decode(p, n=2, type=0, hq=4, q=FAKE, qs=(512, 128), ctx=FAKE, table=FAKE, blocks=4, stride=4, scale=1.0, out=FAKE,
           os=(512, 128), mass_in=None, mass=None, ws=FAKE, size=1 << 40):
    return LIB.peek_decode_attention(None if p is None else ctypes.byref(p), n, type, hq, q, *qs, ctx, table, blocks,
                                     stride, scale, out, *os, None, mass_in, mass, ws, size, None)


def evict(n=2, h=2, block=16, ctx=FAKE, table=FAKE, blocks=4, stride=4, mass=ctypes.c_void_p(0x20000), keep=FAKE,
          sink=0, recent=1, ctx_out=FAKE, table_out=ctypes.c_void_p(0x30000), mass_out=ctypes.c_void_p(0x40000),
          freed=ctypes.c_void_p(0x50000), num=FAKE, ws=FAKE, size=1 << 40):
    return LIB.peek_kv_evict(n, h, block, ctx, table, blocks, stride, mass, keep, sink, recent, ctx_out, table_out,
                             mass_out, freed, num, ws, size, None)


@pytest.mark.parametrize("kw", BAD_POOLS, ids=str)
def test_bad_pools_are_refused(kw):
    p = pool(**kw)
    for call in (append, prefill, decode):
        assert call(p) == BAD
        assert P.peek_last_error()


def test_missing_pool():
    assert append(None) == BAD and decode(None) == BAD
    assert prefill(None) == BAD and "together" in P.peek_last_error()          # a prefix without its pool
    assert prefill(pool(), prefix=None) == BAD


@pytest.mark.parametrize("call", [append, prefill, decode])
def test_shared_refusals(call):
    p = pool()
    for kw in (dict(n=-1), dict(type=2), dict(type=-1), dict(blocks=-1), dict(stride=3), dict(table=None),
               dict(blocks=1 << 28, stride=1 << 28)):
        assert call(p, **kw) == BAD, kw
    first, strides = ("k", "ks") if call is append else ("q", "qs")
    for kw in ({first: None}, {first: ODD}, {strides: (252, 128)}, {strides: (256, 4)}, {strides: (-256, 128)}):
        assert call(p, **kw) == BAD, kw
    assert call(p, n=0, **{first: None}) == P.PEEK_OK


def test_append_refusals():
    p = pool()
    for kw in (dict(tokens=-1), dict(v=None), dict(v=ODD), dict(vs=(256, 4)), dict(off=None), dict(ctx=None),
               dict(tokens=1 << 40)):
        assert append(p, **kw) == BAD, kw
    assert append(p, tokens=0, k=None) == P.PEEK_OK


def test_attention_refusals():
    p = pool()
    for call in (prefill, decode):
        for kw in (dict(hq=3), dict(hq=0), dict(hq=65538), dict(scale=float("nan")), dict(scale=float("inf")),
                   dict(out=None), dict(out=ODD), dict(os=(512, 100))):
            assert call(p, **kw) == BAD, kw
    for kw in (dict(h=4), dict(d=64), dict(d=96), dict(h=0), dict(k=None), dict(v=ODD), dict(off=None),
               dict(tokens=-1), dict(ks=(1 << 23, 128)), dict(vs=(1 << 23, 128))):
        assert prefill(p, **kw) == BAD, kw
    assert decode(p, ctx=None) == BAD
    assert decode(p, mass_in=FAKE) == BAD and "d_mass" in P.peek_last_error()


def test_workspaces():
    p = pool()
    need = LIB.peek_decode_attention_workspace(ctypes.byref(p), 2, 4, 4, 1)
    assert need % 256 == 0
    if need:
        assert decode(p, mass=FAKE, size=need - 1) == P.PEEK_ERR_WORKSPACE_TOO_SMALL
        assert decode(p, mass=FAKE, ws=None) == BAD and decode(p, mass=FAKE, ws=ctypes.c_void_p(0x10010)) == BAD
    assert LIB.peek_decode_attention_workspace(None, 2, 4, 4, 1) == 0
    assert LIB.peek_decode_attention_workspace(ctypes.byref(p), -1, 4, 4, 1) == 0
    need = LIB.peek_prefill_attention_workspace(1, 8, 32, 8, 128, 1 << 16)
    assert need % 256 == 0
    assert LIB.peek_prefill_attention_workspace(-1, 8, 32, 8, 128, 0) == 0
    assert LIB.peek_prefill_attention_workspace(1, 0, 32, 8, 128, 0) == 0


def test_evict_refusals():
    for kw in (dict(n=-1), dict(h=0), dict(h=2000), dict(block=3), dict(block=512), dict(blocks=-1), dict(stride=2),
               dict(ctx=None), dict(table=None), dict(mass=None), dict(keep=None), dict(sink=-1), dict(recent=0),
               dict(ctx_out=None), dict(table_out=None), dict(mass_out=None), dict(freed=None), dict(num=None),
               dict(table_out=FAKE), dict(freed=FAKE), dict(mass_out=ctypes.c_void_p(0x20010))):
        assert evict(**kw) == BAD, kw
    assert evict(n=0, ctx=None) == P.PEEK_OK
    assert LIB.peek_kv_evict_workspace(-1, 2, 4) == 0
    need = LIB.peek_kv_evict_workspace(2, 2, 40000)
    assert need % 256 == 0
    if need:
        far = {k: ctypes.c_void_p(0x10000000 * i) for i, k in
               enumerate(("table", "mass", "table_out", "mass_out", "freed"), 1)}
        assert evict(blocks=40000, stride=40000, size=need - 1, **far) == P.PEEK_ERR_WORKSPACE_TOO_SMALL


def test_binding_refuses_what_the_entry_points_cannot_see():
    pages, scales = torch.zeros(4, 2, 1, 16, 64, dtype=torch.int8), torch.ones(4, 2, 1)
    with pytest.raises(TypeError, match="pages"):
        P.KVPool(pages.float(), scales)
    with pytest.raises(ValueError, match="pages"):
        P.KVPool(pages[0], scales)
    with pytest.raises(ValueError, match="scales"):
        P.KVPool(pages, scales[:3])
    with pytest.raises(ValueError, match="device tensor"):
        P.KVPool(pages, scales)
    q = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device tensor"):
        P._rows(q, "q", torch.bfloat16)
    with pytest.raises(ValueError, match="contiguous"):
        P._rows(q.transpose(1, 2).contiguous().transpose(1, 2), "q", torch.bfloat16)
    with pytest.raises(TypeError, match="q must be"):
        P._rows(q, "q", torch.float16)
    with pytest.raises(TypeError, match="bfloat16 or"):
        P._row_type(q.float(), "q")
    with pytest.raises(ValueError, match="block_table"):
        P._table(torch.zeros(3, 4, dtype=torch.int32), 2)
    with pytest.raises(TypeError, match="block_table"):
        P._table(torch.zeros(2, 4, dtype=torch.int64), 2)
    off = torch.tensor([0, 3])
    with pytest.raises(ValueError, match="together"):
        P.peek_prefill_attention(q, q, q, off, q, None, prefix=torch.zeros(1, dtype=torch.int32))
