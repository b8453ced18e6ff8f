"""Refusals of the entry points for shared prefixes, accumulated weights and eviction: on the host, before a device is touched."""
import ctypes

import pytest

from tests.test_abi import F, LS_EINVAL, LS_ENOMEM, LS_EUNSUPPORTED, LS_OK, lib, pool  # noqa: F401  (fixtures)

P, I32, SZ, FL = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t, ctypes.c_float
LS_EHIP = -5


def no_gpu():
    import torch
    return not torch.cuda.is_available()


def shared(lib, pool, **kw):  # noqa: F811
    a = dict(layer=0, S=6, hq=32, q=F, bt=F, maxb=8, lens=F, G=2, starts=F, M=5, members=F, prefix=F, scale=0.088, out=F, ws=F,
             wsb=1 << 40)
    a.update(kw)
    return lib.paged_attn_decode_shared(pool, a["layer"], a["S"], a["hq"], P(a["q"]), P(a["bt"]), a["maxb"], P(a["lens"]), a["G"],
                                        P(a["starts"]), a["M"], P(a["members"]), P(a["prefix"]), FL(a["scale"]), P(a["out"]),
                                        P(a["ws"]), SZ(a["wsb"]), None)


def weights(lib, pool, **kw):  # noqa: F811
    a = dict(layer=0, S=6, hq=32, q=F, bt=F, maxb=8, lens=F, reused=F, begin=F, first=F, G=2, starts=F, M=5, members=F, prefix=F,
             scale=0.088, out=F, w=F, pos=F, ws=F, wsb=1 << 40)
    a.update(kw)
    return lib.paged_attn_decode_weights(pool, a["layer"], a["S"], a["hq"], P(a["q"]), P(a["bt"]), a["maxb"], P(a["lens"]),
                                         P(a["reused"]), P(a["begin"]), P(a["first"]), a["G"], P(a["starts"]), a["M"],
                                         P(a["members"]), P(a["prefix"]), FL(a["scale"]), P(a["out"]), P(a["w"]), P(a["pos"]),
                                         P(a["ws"]), SZ(a["wsb"]), None)


NONE = dict(G=0, M=0, starts=None, members=None, prefix=None)
BOTH = [
    (dict(layer=2), LS_EINVAL), (dict(layer=-1), LS_EINVAL), (dict(S=-1), LS_EINVAL), (dict(hq=30), LS_EINVAL), (dict(hq=0), LS_EINVAL),
    (dict(hq=64), LS_EUNSUPPORTED), (dict(hq=12), LS_EUNSUPPORTED), (dict(maxb=0), LS_EINVAL), (dict(maxb=16385), LS_EUNSUPPORTED),
    (dict(S=2049), LS_EUNSUPPORTED), (dict(scale=0.0), LS_EINVAL), (dict(scale=float("nan")), LS_EINVAL), (dict(scale=-1.0), LS_EINVAL),
    (dict(q=None), LS_EINVAL), (dict(bt=None), LS_EINVAL), (dict(lens=None), LS_EINVAL), (dict(out=None), LS_EINVAL),
    (dict(ws=None), LS_EINVAL), (dict(q=F + 8), LS_EINVAL), (dict(out=F + 2), LS_EINVAL), (dict(ws=F + 8), LS_EINVAL),
    (dict(bt=F + 2), LS_EINVAL), (dict(lens=F + 1), LS_EINVAL), (dict(G=-1), LS_EINVAL), (dict(M=-1), LS_EINVAL), (dict(G=6), LS_EINVAL),
    (dict(M=7), LS_EINVAL), (dict(starts=None), LS_EINVAL), (dict(members=None), LS_EINVAL), (dict(prefix=None), LS_EINVAL),
    (dict(starts=F + 2), LS_EINVAL), (dict(members=F + 2), LS_EINVAL), (dict(prefix=F + 2), LS_EINVAL), (dict(G=0), LS_EINVAL),
    (dict(G=0, M=0), LS_EINVAL), (dict(NONE, M=1), LS_EINVAL), (dict(wsb=4096), LS_ENOMEM), (dict(NONE, wsb=100), LS_ENOMEM),
    (dict(NONE, S=0), LS_OK),
]


@pytest.mark.parametrize("kw,status", BOTH)
def test_decode_shared_rejects(lib, pool, kw, status):  # noqa: F811
    assert shared(lib, pool, **kw) == status


@pytest.mark.parametrize("kw,status", BOTH + [
    (dict(w=None), LS_EINVAL), (dict(w=F + 4), LS_EINVAL), (dict(pos=None), LS_EINVAL), (dict(pos=F + 8), LS_EINVAL),
    (dict(reused=None), LS_EINVAL), (dict(reused=None, pos=None), LS_EINVAL), (dict(reused=F + 2), LS_EINVAL),
    (dict(begin=F + 2), LS_EINVAL), (dict(first=F + 2), LS_EINVAL),
])
def test_decode_weights_rejects(lib, pool, kw, status):  # noqa: F811
    assert weights(lib, pool, **kw) == status


def test_decodes_take_what_may_be_left_out(lib, pool):  # noqa: F811
    if no_gpu():                                          # past the checks, there is no device to launch on
        assert shared(lib, pool) == LS_EHIP and shared(lib, pool, **NONE) == LS_EHIP
        assert weights(lib, pool, **NONE, begin=None, first=None) == LS_EHIP
        assert weights(lib, pool, reused=None, begin=None, pos=None) == LS_EHIP


def test_workspace_sizes(lib, pool):  # noqa: F811
    f, g = lib.ls_decode_shared_workspace_bytes, lib.ls_decode_weights_workspace_bytes
    f.restype = g.restype = SZ
    assert 0 < f(pool, 1, 32, 0, 0) < f(pool, 64, 32, 0, 0) < f(pool, 64, 32, 1, 64) < f(pool, 64, 32, 8, 64)
    assert g(pool, 64, 32, 1, 64) >= f(pool, 64, 32, 1, 64) + 100 * 32 * 64             # the pool has 100 blocks
    for bad in ((0, 32, 0, 0), (2049, 32, 0, 0), (64, 30, 0, 0), (64, 0, 0, 0), (64, 32, -1, 0), (64, 32, 3, 2), (64, 32, 1, 65), (64, 32, 0, 1)):
        assert f(pool, *bad) == 0 and g(pool, *bad) == 0
    assert f(None, 1, 32, 0, 0) == 0 == g(None, 1, 32, 0, 0)
    h = lib.ls_weights_prefill_workspace_bytes
    h.restype = SZ
    assert 0 < h(pool, 4, 32, 100, 30, 1, 8) < h(pool, 4, 32, 100, 30, 16, 8) < h(pool, 4, 32, 100, 30, 16, 800)
    assert h(pool, 4, 32, 100, 30, 16, 8) == h(pool, 4, 32, 3000, 30, 16, 8)
    assert h(pool, 4, 32, 2**31 - 1, 2**31 - 1, 2**31 - 1, 8) == h(pool, 4, 32, 200, 128, 128, 8)      # a turn fits its table
    for bad in ((0, 32, 10, 5, 1, 8), (2049, 32, 10, 5, 1, 8), (4, 30, 10, 5, 1, 8), (4, 32, 10, 11, 1, 8), (4, 32, 10, 0, 1, 8),
                (4, 32, 10, 5, 0, 8), (4, 32, 10, 5, 1, 0), (4, 32, 10, 5, 1, 16385)):
        assert h(pool, *bad) == 0
    assert h(None, 4, 32, 10, 5, 1, 8) == 0


def prompt(lib, pool, **kw):  # noqa: F811
    a = dict(layer=0, S=2, hq=32, q=F, cu=F, ctx=F, total=40, longest=30, bt=F, maxb=8, rows=16, begin=F, first=F, scale=0.088, w=F,
             pos=F, ws=F, wsb=1 << 40)
    a.update(kw)
    return lib.kv_weights_prefill(pool, a["layer"], a["S"], a["hq"], P(a["q"]), P(a["cu"]), P(a["ctx"]), a["total"], a["longest"],
                                  P(a["bt"]), a["maxb"], a["rows"], P(a["begin"]), P(a["first"]), FL(a["scale"]), P(a["w"]),
                                  P(a["pos"]), P(a["ws"]), SZ(a["wsb"]), None)


@pytest.mark.parametrize("kw,status", [
    (dict(layer=2), LS_EINVAL), (dict(S=-1), LS_EINVAL), (dict(hq=30), LS_EINVAL), (dict(hq=64), LS_EUNSUPPORTED), (dict(maxb=0), LS_EINVAL),
    (dict(maxb=16385), LS_EUNSUPPORTED), (dict(S=2049), LS_EUNSUPPORTED), (dict(scale=0.0), LS_EINVAL), (dict(total=-1), LS_EINVAL),
    (dict(longest=-1), LS_EINVAL), (dict(longest=41), LS_EINVAL), (dict(rows=0), LS_EINVAL), (dict(rows=-4), LS_EINVAL),
    (dict(q=None), LS_EINVAL), (dict(cu=None), LS_EINVAL), (dict(ctx=None), LS_EINVAL), (dict(bt=None), LS_EINVAL),
    (dict(w=None), LS_EINVAL), (dict(pos=None), LS_EINVAL), (dict(ws=None), LS_EINVAL), (dict(q=F + 8), LS_EINVAL),
    (dict(w=F + 4), LS_EINVAL), (dict(pos=F + 4), LS_EINVAL), (dict(ws=F + 8), LS_EINVAL), (dict(cu=F + 2), LS_EINVAL),
    (dict(ctx=F + 2), LS_EINVAL), (dict(bt=F + 2), LS_EINVAL), (dict(begin=F + 2), LS_EINVAL), (dict(first=F + 2), LS_EINVAL),
    (dict(wsb=1000), LS_ENOMEM), (dict(S=0), LS_OK), (dict(total=0, longest=0, q=None), LS_OK),
])
def test_weights_prefill_rejects(lib, pool, kw, status):  # noqa: F811
    assert prompt(lib, pool, **kw) == status


# (the pool has 2 layers of 100 blocks of 4 KV heads: 51200 bytes an entry array)
W0, W1, P0, P1 = F + 0x100000, F + 0x200000, F + 0x300000, F + 0x400000


def evict(lib, pool, **kw):  # noqa: F811
    a = dict(lb=0, lc=2, S=4, lens=F, bt=F + 0x1000, maxb=8, budget=50, limit=60, recent=10, first=F + 0x100, nextp=F + 0x200, w=W0, pos=P0,
             wn=W1, pn=P1, nextl=F + 0x300, ring=F + 0x2000, size=100, counts=F + 0x400, after=F + 0x500)
    a.update(kw)
    return lib.kv_evict(pool, a["lb"], a["lc"], a["S"], P(a["lens"]), P(a["bt"]), a["maxb"], a["budget"], a["limit"], a["recent"],
                        P(a["first"]), P(a["nextp"]), P(a["w"]), P(a["pos"]), P(a["wn"]), P(a["pn"]), P(a["nextl"]), P(a["ring"]),
                        a["size"], P(a["counts"]), P(a["after"]), None)


@pytest.mark.parametrize("kw", [
    dict(lb=-1), dict(lb=1), dict(lc=0), dict(lc=3), dict(lb=2, lc=1), dict(S=-1), dict(maxb=0), dict(maxb=-7), dict(budget=0),
    dict(limit=49), dict(recent=-1), dict(recent=51), dict(lens=None), dict(bt=None), dict(nextp=None), dict(w=None), dict(pos=None),
    dict(wn=None), dict(pn=None), dict(nextl=None), dict(ring=None), dict(size=0), dict(counts=None), dict(after=None),
    dict(ring=None, size=0), dict(wn=W0), dict(pn=P0), dict(w=W0 + 4), dict(pn=P1 + 8), dict(lens=F + 2), dict(counts=F + 0x404),
    dict(ring=F + 0x2002), dict(nextl=F), dict(nextl=F + 4), dict(nextl=F + 0x100), dict(nextl=F + 0x208), dict(ring=F + 0x1000),
    dict(wn=W0 + 16), dict(wn=P0), dict(pn=W0 + 51184), dict(pn=W1), dict(after=F + 0x408), dict(nextl=F + 0x500), dict(nextp=W1 + 100),
    dict(bt=P1 - 4), dict(ring=W0),
])
def test_evict_rejects(lib, pool, kw):  # noqa: F811
    assert evict(lib, pool, **kw) == LS_EINVAL


def test_limits_of_the_schedule(lib):  # noqa: F811
    from tests.test_abi import _desc
    h = ctypes.c_void_p()
    for heads, status in ((32, LS_EUNSUPPORTED), (31, LS_ENOMEM)):
        d = _desc(num_layers=1, num_kv_heads=heads, num_blocks=1, kv_bytes=1 << 30)
        assert lib.kv_pool_create(ctypes.byref(d), ctypes.byref(h)) == LS_OK
        big = dict(S=2048, maxb=16384, hq=heads, wsb=1000, M=2048)           # sessions x blocks x KV heads: 2^30, and less
        assert shared(lib, h, **big) == status
        assert weights(lib, h, **big) == status
        assert prompt(lib, h, S=2048, maxb=16384, hq=heads, wsb=1000) == status
        lib.kv_pool_destroy(h)


def test_evict_limits(lib, pool):  # noqa: F811
    assert evict(lib, pool, maxb=16385, bt=F + 0x10000000) == LS_EUNSUPPORTED
    assert evict(lib, pool, S=(1 << 20) + 1) == LS_EUNSUPPORTED


def test_evict_takes_arrays_in_place_and_no_ring(lib, pool):  # noqa: F811
    if no_gpu():
        assert evict(lib, pool) == LS_EHIP
        assert evict(lib, pool, wn=W0, pn=P0, after=F + 0x400) == LS_EHIP
        assert evict(lib, pool, ring=None, size=0, counts=None, after=None, first=None, lb=1, lc=1) == LS_EHIP
        assert evict(lib, pool, S=0, lens=None, bt=None, nextp=None, nextl=None) == LS_EHIP      # (counters are still written)
