"""Host-only checks of the calls around a decode step: rotary frequencies, what the calls refuse before any GPU work,
and how much scratch they ask for. Fake device pointers are never read."""
import ctypes
import math

import numpy as np
import pytest

import paper_2607_02525_amd as P
from tests.test_attention_args import BAD, BAD_POOLS, FAKE, ODD, decode, pool

torch = pytest.importorskip("torch")
LIB = P._lib
SMALL = P.PEEK_ERR_WORKSPACE_TOO_SMALL


def ref(p):
    return None if p is None else ctypes.byref(p)


def rotary(**kw):
    f = dict(d_freq=0x10000, rot_dim=128, interleaved=0, magnitude=1.0, eps=1e-6, d_q_norm=None, d_k_norm=None)
    f.update(kw)
    return P._RotaryStruct(*(f[k] for k, _ in P._RotaryStruct._fields_))


def rotate(p, n=2, tokens=3, type=0, hq=4, h=2, d=128, rot=None, q=FAKE, qs=(512, 128), k=FAKE, ks=(256, 128), v=FAKE,
           vs=(256, 128), off=FAKE, ctx=FAKE, table=FAKE, blocks=4, stride=4, qo=FAKE, qos=(512, 128), ko=FAKE,
           kos=(256, 128)):
    rot = rotary() if rot is None else rot
    return LIB.peek_rotate_append(ref(p), n, tokens, type, hq, h, d, ref(rot) if rot != 0 else None, q, *qs, k, *ks, v,
                                  *vs, off, ctx, table, blocks, stride, qo, *qos, ko, *kos, None)


def read(p, n=2, tokens=3, type=0, off=FAKE, first=FAKE, table=FAKE, blocks=4, stride=4, k=FAKE, ks=(256, 128), v=FAKE,
         vs=(256, 128)):
    return LIB.peek_kv_read(ref(p), n, tokens, type, off, first, table, blocks, stride, k, *ks, v, *vs, None)


def shared(p, n=2, type=0, hq=4, q=FAKE, qs=(512, 128), ctx=FAKE, table=FAKE, blocks=4, stride=4, groups=1,
           members=FAKE, offsets=FAKE, tokens=FAKE, scale=1.0, out=FAKE, os=(512, 128), ws=FAKE, size=1 << 40):
    return LIB.peek_shared_decode_attention(ref(p), n, type, hq, q, *qs, ctx, table, blocks, stride, groups, members,
                                            offsets, tokens, scale, out, *os, None, ws, size, None)


def bounds(p, n=2, first=None, ctx=FAKE, table=FAKE, blocks=4, stride=4, out=FAKE):
    return LIB.peek_kv_bounds(ref(p), n, first, ctx, table, blocks, stride, out, None)


def select(p, b=FAKE, n=2, type=0, hq=4, q=FAKE, qs=(512, 128), ctx=FAKE, table=FAKE, blocks=8, stride=8, keep=4,
           sink=1, recent=1, ctx_out=FAKE, table_out=FAKE, ws=FAKE, size=1 << 40):
    return LIB.peek_block_select(ref(p), b, n, type, hq, q, *qs, ctx, table, blocks, stride, keep, sink, recent,
                                 ctx_out, table_out, ws, size, None)


def sparse(p, n=2, type=0, hq=4, q=FAKE, qs=(512, 128), ctx=FAKE, table=FAKE, keep=4, scale=1.0, out=FAKE,
           os=(512, 128), ws=FAKE, size=1 << 40):
    return LIB.peek_sparse_decode_attention(ref(p), n, type, hq, q, *qs, ctx, table, keep, scale, out, *os, None, ws,
                                            size, None)


@pytest.mark.parametrize("kw", BAD_POOLS, ids=str)
def test_bad_pools_are_refused(kw):
    for call in (rotate, read, shared, bounds, select, sparse):
        assert call(pool(**kw)) == BAD and P.peek_last_error()


ROWS = [dict(ks=(255, 128)), dict(ks=(-8, 128)), dict(k=ODD), dict(k=None)]
REFUSED = [
    (rotate, [dict(n=-1), dict(tokens=-1), dict(type=2), dict(hq=-1), dict(hq=65537), dict(h=0), dict(h=1025), dict(h=4),
              dict(d=96), dict(d=64), dict(rot=0), dict(rot=rotary(rot_dim=8)), dict(rot=rotary(rot_dim=-16)),
              dict(rot=rotary(rot_dim=144)), dict(rot=rotary(d_freq=None)), dict(rot=rotary(magnitude=math.inf)),
              dict(rot=rotary(magnitude=math.nan)), dict(rot=rotary(eps=-1.0)), dict(rot=rotary(eps=math.nan)),
              dict(rot=rotary(d_freq=0x10004)), dict(rot=rotary(d_q_norm=0x10008)), dict(rot=rotary(d_k_norm=0x10002)), dict(q=None), dict(qo=None),
              dict(qos=(256, 128)), dict(qos=(512, 64)), dict(kos=(128, 128)), dict(ko=ODD), dict(v=None), dict(v=ODD),
              dict(off=None), dict(ctx=None), dict(table=None), dict(stride=3), dict(blocks=-1),
              dict(tokens=1 << 40), *ROWS]),
    (read, [dict(n=-1), dict(tokens=-1), dict(type=3), dict(off=None), dict(first=None), dict(table=None),
            dict(stride=3), dict(v=None), dict(v=ODD), dict(ks=(128, 128)), dict(vs=(256, 64)), dict(tokens=1 << 40),
            *ROWS]),
    (shared, [dict(n=-1), dict(groups=-1), dict(groups=1 << 24), dict(type=2), dict(hq=3), dict(hq=0), dict(scale=math.nan), dict(q=None),
              dict(qs=(4, 128)), dict(ctx=None), dict(table=None), dict(stride=3), dict(offsets=None),
              dict(tokens=None), dict(out=None), dict(os=(256, 128)), dict(ws=None), dict(ws=ODD), dict(n=1 << 24),
              dict(blocks=1 << 28, stride=1 << 28)]),
    (bounds, [dict(n=-1), dict(ctx=None), dict(table=None), dict(stride=3), dict(out=None), dict(out=ODD)]),
    (select, [dict(b=None), dict(b=ODD), dict(n=-1), dict(type=2), dict(hq=3), dict(q=None), dict(ctx=None),
              dict(table=None), dict(stride=3), dict(keep=0), dict(sink=-1), dict(recent=0), dict(sink=4),
              dict(sink=2, recent=3), dict(keep=1 << 28), dict(ctx_out=None), dict(table_out=None), dict(ws=None),
              dict(ws=ODD), dict(sink=(1 << 31) - 1, recent=(1 << 31) - 1)]),
    (sparse, [dict(n=-1), dict(type=2), dict(hq=3), dict(q=None), dict(ctx=None), dict(table=None), dict(keep=-1),
              dict(scale=math.inf), dict(out=None), dict(os=(256, 128)), dict(keep=1 << 28)]),
]


@pytest.mark.parametrize("call,kw", [(c, kw) for c, all_ in REFUSED for kw in all_],
                         ids=[f"{c.__name__} {i} {'+'.join(kw)}" for c, all_ in REFUSED for i, kw in enumerate(all_)])
def test_refusals(call, kw):
    assert call(pool(), **kw) == BAD
    assert P.peek_last_error()


def test_refusals_without_a_pool():
    assert rotate(None, v=FAKE, table=None) == BAD
    assert rotate(None, v=None, table=FAKE) == BAD
    assert rotate(None, v=None, table=None, ko=None) == BAD           # k for nothing
    for call in (read, shared, bounds, select, sparse):
        assert call(None) == BAD


def test_nothing_to_do_is_fine():
    for kw in (dict(n=0), dict(tokens=0), dict(n=0, tokens=0, off=None, ctx=None)):
        assert rotate(pool(), **kw) == P.PEEK_OK
    assert read(pool(), n=0) == P.PEEK_OK and read(pool(), tokens=0) == P.PEEK_OK
    assert shared(pool(), n=0, q=None, out=None) == P.PEEK_OK
    assert bounds(pool(), n=0) == P.PEEK_OK and bounds(pool(), blocks=0, stride=0) == P.PEEK_OK
    assert select(pool(), n=0) == P.PEEK_OK and sparse(pool(), n=0) == P.PEEK_OK


def test_workspaces():
    p, byref = pool(), ctypes.byref(pool())
    assert LIB.peek_shared_decode_attention_workspace(None, 2, 4, 4, 1) == 0
    assert LIB.peek_shared_decode_attention_workspace(byref, 2, 3, 4, 1) == 0
    assert LIB.peek_block_select_workspace(byref, -1, 4) == 0
    for n, blocks, groups in ((1, 4, 1), (64, 500, 8), (3, 100000, 0), (200, 1, 200)):
        need = LIB.peek_shared_decode_attention_workspace(byref, n, 4, blocks, groups)
        assert need % 256 == 0 and need > 0
        kw = dict(n=n, blocks=blocks, stride=blocks, groups=groups)
        assert shared(p, size=need - 1, **kw) == SMALL
        need = LIB.peek_block_select_workspace(byref, n, blocks)
        assert need >= n * 2 * blocks * 4
        assert select(p, n=n, blocks=blocks, stride=blocks, size=need - 1) == SMALL
    need = LIB.peek_sparse_decode_attention_workspace(byref, 2, 4, 4096)
    assert need > 0 and sparse(p, keep=4096, size=need - 1) == SMALL


# -------------------------------------------------------------- frequencies
def test_frequencies():
    d, base, s, T = 64, 10000.0, 8.0, 4096.0
    f = np.array([base ** (-2 * i / d) for i in range(d // 2)])
    same = dict(rtol=1e-14, atol=0)
    np.testing.assert_allclose(P.peek_rotary_frequencies(d, base), f, **same)
    np.testing.assert_allclose(P.peek_rotary_frequencies(d, base, P.PEEK_ROTARY_LINEAR, s), f / s, **same)
    longer = base * s ** (d / (d - 2))
    np.testing.assert_allclose(P.peek_rotary_frequencies(d, base, P.PEEK_ROTARY_BASE, s),
                               [longer ** (-2 * i / d) for i in range(d // 2)], **same)
    # the slowest pair's wave is s times as long, the fastest as it was
    got = P.peek_rotary_frequencies(d, base, P.PEEK_ROTARY_BASE, s)
    np.testing.assert_allclose([got[0], got[-1]], [f[0], f[-1] / s], rtol=1e-12)
    turns = T * f / (2 * math.pi)
    g = np.clip((turns - 1) / 3, 0, 1)
    got = P.peek_rotary_frequencies(d, base, P.PEEK_ROTARY_TURNS, s, T, 1.0, 4.0)
    np.testing.assert_allclose(got, f * g + f / s * (1 - g), rtol=1e-12)
    assert got[0] == f[0] and abs(got[-1] - f[-1] / s) < 1e-18

    def pair(t):
        return d * math.log(T / (t * 2 * math.pi)) / (2 * math.log(base))
    a, b = max(math.floor(pair(32.0)), 0), min(math.ceil(pair(1.0)), d - 1)
    g = 1 - np.clip((np.arange(d // 2) - a) / (b - a), 0, 1)
    got = P.peek_rotary_frequencies(d, base, P.PEEK_ROTARY_RAMP, s, T, 1.0, 32.0)
    np.testing.assert_allclose(got, f * g + f / s * (1 - g), rtol=1e-12)


@pytest.mark.parametrize("args", [(0, 1e4), (3, 1e4), (130, 1e4), (-2, 1e4), (64, 0.0), (64, -1.0), (64, math.inf),
                                  (64, 1e4, 5), (64, 1e4, -1), (64, 1e4, 1, 0.0), (64, 1e4, 1, math.nan),
                                  (2, 1e4, 2, 2.0), (64, 1e4, 3, 2.0, 0.0), (64, 1e4, 3, 2.0, 100.0, 4.0, 4.0),
                                  (64, 1e4, 4, 2.0, 100.0, 0.0, 4.0), (64, 1.0, 4, 2.0, 100.0, 1.0, 4.0)], ids=str)
def test_frequencies_refused(args):
    with pytest.raises(P.PeekError) as e:
        P.peek_rotary_frequencies(*args)
    assert e.value.status == BAD


# ---------------------------------------------------------------- binding
def test_the_binding_refuses_other_shapes_and_types():
    f16, i32 = torch.float16, torch.int32
    k = torch.zeros(3, 2, 64, dtype=f16)
    at, ctx = torch.zeros(2, dtype=torch.int64), torch.zeros(1, dtype=i32)
    for kw in (dict(q=k), dict(q_out=k), dict(k_out=None), dict(v=k), dict(block_table=torch.zeros(1, 1, dtype=i32))):
        args = dict(q=None, k=k, v=None, offsets=at, context=ctx, freq=None, q_out=None, k_out=k)
        args.update(kw)
        with pytest.raises(ValueError):
            P.peek_rotate_append(**args)
    with pytest.raises(TypeError):
        P.peek_rotate_append(None, k.float(), None, at, ctx, None, None, k_out=k)
    with pytest.raises(ValueError, match="must be"):
        P._exact_arg(torch.zeros(3, 4), "x", torch.float32, 4, 3)
    with pytest.raises(TypeError, match="must be"):
        P._exact_arg(torch.zeros(4, 3), "x", torch.float16, 4, 3)


def test_the_binding_takes_queries_alone_and_refuses_neither():
    f16, i32 = torch.float16, torch.int32
    q = torch.zeros(3, 2, 64, dtype=f16)
    at, ctx = torch.zeros(2, dtype=torch.int64), torch.zeros(1, dtype=i32)
    with pytest.raises(ValueError, match="k and q"):
        P.peek_rotate_append(None, None, None, at, ctx, None, None)
    with pytest.raises(ValueError, match="k must be given"):
        P.peek_rotate_append(q, None, None, at, ctx, None, q, k_out=q)
    with pytest.raises(TypeError, match="float32"):
        P.peek_rotate_append(q.float(), None, None, at, ctx, None, q.float())
    # as far as the tensors' place, which is not a GPU here
    with pytest.raises(Exception, match="GPU|CUDA|cuda|device"):
        P.peek_rotate_append(q, None, None, at, ctx, None, q)


# ------------------------------------------------- launches of 2^32 threads or more
def test_rotations_that_no_launch_can_hold_are_refused():
    """Workgroups of one launch times their threads stay below 2^32, whichever of its parts they are for."""
    small = dict(kv_heads=1, block_size=4, head_dim=64)
    one = dict(h=1, d=64, ks=(64, 64), vs=(64, 64), kos=(64, 64), qs=(64, 64), qos=(64, 64), hq=1)
    # 14 million blocks' workgroups (K and V) beside 7 million of four rows each
    assert rotate(pool(**small), tokens=28_000_000, rot=rotary(rot_dim=64), **one) == BAD
    assert "too many" in P.peek_last_error()


def test_decodes_that_no_launch_can_hold_are_refused():
    # own keys' workgroups and those of shared keys beside them
    wide = dict(qs=(64, 64), os=(64, 64), hq=1)
    most = (1 << 24) - 1
    assert shared(pool(kv_heads=1, block_size=16, head_dim=64), n=most, blocks=1, stride=1, groups=1, size=1 << 50,
                  **wide) == BAD
    assert "too many" in P.peek_last_error()
    # joins by 16 wavefronts to a row: 2^22 rows
    heads = dict(n=24576, hq=256, qs=(256 * 64, 64), os=(256 * 64, 64), size=1 << 60)
    width = dict(blocks=8192, stride=8192)
    for call, kw in ((shared, width), (decode, width), (sparse, dict(keep=8192))):
        assert call(pool(kv_heads=1, block_size=16, head_dim=64), **kw, **heads) == BAD
        assert "too many" in P.peek_last_error()


def test_choices_that_no_launch_can_hold_are_refused():
    # choices by 16 wavefronts to a (sequence, kv head)
    assert select(pool(kv_heads=1024, block_size=4, head_dim=64), n=4096, hq=1024, qs=(1024 * 64, 64), blocks=5000,
                  stride=5000, size=1 << 60) == BAD
    assert "too many" in P.peek_last_error()
