"""Refusals of the windowed entry points, kv_tables_update and kv_append: on the host, before a device is touched."""
import ctypes

import numpy as np
import pytest

from tests.test_abi import F, LS_EINVAL, LS_ENOMEM, LS_EUNSUPPORTED, LS_OK, Desc, _desc, lib, pool  # noqa: F401  (fixtures)

P, I32, I64, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
LS_EHIP = -5


def i32s(v):
    return None if v is None else (I32 * len(v))(*v)


def decode(lib, pool, **kw):  # noqa: F811
    a = dict(layer=0, S=4, hq=32, q=F, kn=None, vn=None, bt=F, maxb=8, lens=F, host=None, W=64, sinks=4, scale=0.088, out=F,
             ws=F, wsb=1 << 30)
    a.update(kw)
    return lib.paged_attn_decode_window(pool, a["layer"], a["S"], a["hq"], P(a["q"]), P(a["kn"]), P(a["vn"]), P(a["bt"]), a["maxb"],
                                        P(a["lens"]), i32s(a["host"]), a["W"], a["sinks"], ctypes.c_float(a["scale"]), P(a["out"]),
                                        P(a["ws"]), SZ(a["wsb"]), None)


@pytest.mark.parametrize("kw,status", [
    (dict(W=0), LS_EINVAL), (dict(W=-5), LS_EINVAL), (dict(W=(1 << 29) + 1), LS_EINVAL), (dict(sinks=-1), LS_EINVAL),
    (dict(sinks=(1 << 29) + 1), LS_EINVAL), (dict(maxb=1 << 27), LS_EINVAL), (dict(layer=2), LS_EINVAL), (dict(hq=30), LS_EINVAL),
    (dict(hq=64), LS_EUNSUPPORTED), (dict(q=None), LS_EINVAL), (dict(q=F + 8), LS_EINVAL), (dict(out=F + 2), LS_EINVAL),
    (dict(kn=F, vn=F + 4), LS_EINVAL), (dict(kn=F), LS_EINVAL), (dict(ws=F + 8), LS_EINVAL), (dict(bt=F + 2), LS_EINVAL),
    (dict(lens=F + 1), LS_EINVAL), (dict(maxb=0), LS_EINVAL), (dict(scale=0.0), LS_EINVAL), (dict(scale=float("nan")), LS_EINVAL),
    (dict(wsb=16), LS_ENOMEM), (dict(S=2049), LS_EUNSUPPORTED), (dict(S=-1), LS_EINVAL), (dict(W=1 << 29, maxb=20000), LS_EUNSUPPORTED),
    (dict(host=[0, 1, 1, 1]), LS_EINVAL), (dict(host=[1, 1, 1, 129]), LS_EINVAL), (dict(S=0), LS_OK),
])
def test_decode_window_rejects(lib, pool, kw, status):  # noqa: F811
    assert decode(lib, pool, **kw) == status


def test_window_bounds_the_workspace_and_the_table(lib, pool):  # noqa: F811
    f = lib.ls_decode_window_workspace_bytes
    f.restype = SZ
    lib.ls_decode_workspace_bytes.restype = SZ
    wide = f(pool, 64, 32, 100000, 1024, 4)
    assert 0 < wide == f(pool, 64, 32, 67, 1024, 4) == f(pool, 64, 32, 1 << 26, 1024, 4)      # 65 blocks of a window, 1 of sinks ...
    assert f(pool, 64, 32, 16, 1024, 4) < wide
    for bad in ((0, 4), (-1, 0), (16, -1), ((1 << 29) + 1, 0)):
        assert f(pool, 64, 32, 100, *bad) == 0
    assert f(None, 64, 32, 100, 64, 0) == 0 and f(pool, 64, 32, 0, 64, 0) == 0
    # a table far past the limit of blocks with seen keys passes the checks; without a GPU the launch is what fails
    import torch
    if not torch.cuda.is_available():
        assert decode(lib, pool, maxb=1 << 20) == LS_EHIP


def prefill(lib, pool, **kw):  # noqa: F811
    a = dict(layer=0, S=2, hq=32, q=F, kn=None, vn=None, cu=F, ctx=F, host=None, total=40, longest=30, bt=F, maxb=8, W=64, sinks=4,
             scale=0.088, out=F, ws=None, wsb=0)
    a.update(kw)
    return lib.paged_attn_prefill_window(pool, a["layer"], a["S"], a["hq"], P(a["q"]), P(a["kn"]), P(a["vn"]), P(a["cu"]), P(a["ctx"]),
                                         i32s(a["host"]), a["total"], a["longest"], P(a["bt"]), a["maxb"], a["W"], a["sinks"],
                                         ctypes.c_float(a["scale"]), P(a["out"]), P(a["ws"]), SZ(a["wsb"]), None)


@pytest.mark.parametrize("kw,status", [
    (dict(W=0), LS_EINVAL), (dict(W=(1 << 29) + 1), LS_EINVAL), (dict(sinks=-1), LS_EINVAL), (dict(maxb=1 << 27), LS_EINVAL),
    (dict(q=F + 8), LS_EINVAL), (dict(out=None), LS_EINVAL), (dict(out=F + 8), LS_EINVAL), (dict(kn=F + 2, vn=F), LS_EINVAL),
    (dict(kn=F), LS_EINVAL), (dict(cu=F + 2), LS_EINVAL), (dict(ctx=F + 2), LS_EINVAL), (dict(longest=41), LS_EINVAL),
    (dict(scale=-1.0), LS_EINVAL), (dict(ws=F, wsb=100), LS_ENOMEM), (dict(ws=F + 8, wsb=1 << 20), LS_EINVAL),
    (dict(host=[30, 5, 10, 200]), LS_EINVAL), (dict(host=[30, 5, 11, 5]), LS_EINVAL), (dict(hq=12), LS_EUNSUPPORTED),
    (dict(total=0, longest=0), LS_OK), (dict(S=0), LS_OK),
])
def test_prefill_window_rejects(lib, pool, kw, status):  # noqa: F811
    assert prefill(lib, pool, **kw) == status


def tables(lib, pool, **kw):  # noqa: F811
    a = dict(S=4, lens=F, new=F + 0x100, bt=F + 0x1000, maxb=8, ring=F + 0x2000, size=100, counts=F + 0x200, after=F + 0x300, W=16,
             sinks=0, total=9, longest=5, next=F + 0x400, cu=F + 0x500, reused=None, slots=F + 0x3000)
    a.update(kw)
    return lib.kv_tables_update(pool, a["S"], P(a["lens"]), P(a["new"]), P(a["bt"]), a["maxb"], P(a["ring"]), a["size"], P(a["counts"]),
                                P(a["after"]), a["W"], a["sinks"], a["total"], a["longest"], P(a["next"]), P(a["cu"]), P(a["reused"]),
                                P(a["slots"]), None)


@pytest.mark.parametrize("kw", [
    dict(S=-1), dict(total=-1), dict(longest=-1), dict(maxb=0), dict(maxb=1 << 27), dict(lens=None), dict(new=None), dict(bt=None),
    dict(next=None), dict(cu=None), dict(slots=None), dict(size=0), dict(size=-3), dict(counts=None), dict(after=None), dict(W=-1),
    dict(W=(1 << 29) + 1), dict(sinks=-1), dict(sinks=(1 << 29) + 1), dict(ring=None), dict(ring=None, size=0, counts=None, after=None),
    dict(ring=None, size=0, counts=None, W=0), dict(lens=F + 2), dict(ring=F + 1), dict(slots=F + 4), dict(counts=F + 4),
    dict(reused=F + 2), dict(total=2**31 - 1), dict(next=F + 4), dict(next=F - 4), dict(after=F + 0x208), dict(reused=F), dict(cu=F + 0x40c),
    dict(reused=F + 0x400), dict(slots=F + 0x2000 + 396), dict(ring=F + 0x1000), dict(new=F), dict(bt=F + 0x2000 - 124),
])
def test_tables_update_rejects(lib, pool, kw):  # noqa: F811
    assert tables(lib, pool, **kw) == LS_EINVAL


def test_tables_update_takes_lengths_and_counters_in_place(lib, pool):  # noqa: F811
    import torch
    if not torch.cuda.is_available():                  # past the checks, there is no device to launch on
        assert tables(lib, pool, next=F, after=F + 0x200) == LS_EHIP
        assert tables(lib, pool, ring=None, size=0, counts=None, after=None, W=0, reused=F + 0x600) == LS_EHIP


def test_tables_update_of_no_sessions_compares_no_empty_arrays(lib, pool):  # noqa: F811
    import torch
    if not torch.cuda.is_available():
        assert tables(lib, pool, S=0, lens=F + 0x2010, new=F + 0x3008, bt=F + 0x2020, next=F + 0x2010) == LS_EHIP


def append(lib, pool, **kw):  # noqa: F811
    a = dict(layer=0, T=4, k=F, v=F, ks=512, vs=512, slots=F, host=None)
    a.update(kw)
    host = None if a["host"] is None else (I64 * len(a["host"]))(*a["host"])
    return lib.kv_append(pool, a["layer"], a["T"], P(a["k"]), P(a["v"]), I64(a["ks"]), I64(a["vs"]), P(a["slots"]), host, None)


@pytest.mark.parametrize("kw,status", [
    (dict(layer=2), LS_EINVAL), (dict(layer=-1), LS_EINVAL), (dict(T=-1), LS_EINVAL), (dict(T=0, k=None, v=None, slots=None), LS_OK),
    (dict(k=None), LS_EINVAL), (dict(v=None), LS_EINVAL), (dict(slots=None), LS_EINVAL), (dict(ks=504), LS_EINVAL), (dict(vs=516), LS_EINVAL),
    (dict(ks=-512), LS_EINVAL), (dict(ks=1 << 62), LS_EINVAL), (dict(k=F + 8), LS_EINVAL), (dict(v=F + 2), LS_EINVAL), (dict(slots=F + 4), LS_EINVAL),
    (dict(host=[0, 1, 2, 1600]), LS_EINVAL), (dict(host=[0, 1, 7, 1]), LS_EINVAL),
])
def test_append_rejects(lib, pool, kw, status):  # noqa: F811
    assert append(lib, pool, **kw) == status


def test_binding_checks_tensors(built_lib):
    import torch
    from paper_2606_22983_amd import kv
    t = torch.zeros(3, dtype=torch.int32)
    for bad in (t, t.long()):
        with pytest.raises(ValueError):
            kv._vector(bad, "seq_lens", 3, (torch.int32,))
    rows = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        kv._rows(rows, "k_new", (4, 2, 64))            # not on a device
    with pytest.raises(ValueError):
        kv._rows(rows, "k_new", (4, 3, 64))
    with pytest.raises(ValueError):
        kv._rows(rows.float(), "k_new", (4, 2, 64))
    assert np.int32(kv.LS_DEVERR_FREE_LIST) == 8


def test_oracle_window_and_tables_by_hand(oracle_lib):
    """The windowed oracle against the plain one where they agree, and a step worked out by hand."""
    rng = np.random.default_rng(0)
    pool_ = rng.integers(0x3C00, 0x4000, (1, 6, 2, 1, 16 * 64), dtype=np.uint16)
    q = rng.integers(0x3C00, 0x4000, (1, 2, 64), dtype=np.uint16)
    bt = np.array([[3, 1, 4, 0]], dtype=np.int32)
    full = oracle_lib.attend(pool_, 16, 64, 0, q, bt, [0], [50], [0], 0.125)
    for w, k in ((50, 0), (1 << 29, 0), (30, 20), (1, 1 << 29)):
        out, mass, score = oracle_lib.attend_window(pool_, 16, 64, 0, q, bt, [0], [49], [0], 0.125, w, k)
        assert np.allclose(out, full, rtol=1e-13) and (mass >= np.abs(out) - 1e-12).all() and (score > 0).all()
    # one key: its own V
    out, _, _ = oracle_lib.attend_window(pool_, 16, 64, 0, q, bt, [0], [33], [0], 0.125, 1, 0)
    from paper_2606_22983_amd import workloads as W
    assert np.array_equal(out[0, 0], W.from_bf16(pool_[0, 4, 1, 0].reshape(64, 16)[:, 1]).astype(np.float64))
    # two keys, 0 and 33
    out, _, _ = oracle_lib.attend_window(pool_, 16, 64, 0, q, bt, [0], [33], [0], 0.125, 1, 1)
    k0 = W.from_bf16(pool_[0, 3, 0, 0].reshape(8, 16, 8)[:, 0].reshape(-1)).astype(np.float64)
    k33 = W.from_bf16(pool_[0, 4, 0, 0].reshape(8, 16, 8)[:, 1].reshape(-1)).astype(np.float64)
    qf = W.from_bf16(q[0, 0]).astype(np.float64)
    w0 = 1 / (1 + np.exp(0.125 * (qf @ k33 - qf @ k0)))
    v0, v33 = (W.from_bf16(pool_[0, b, 1, 0].reshape(64, 16)[:, o]).astype(np.float64) for b, o in ((3, 0), (4, 1)))
    assert np.allclose(out[0, 0], w0 * v0 + (1 - w0) * v33, rtol=1e-12)
    # 30 + 3 tokens: one block opened (position 32); 47 + 2: one (48), and with a window of 16 and 4
    # first tokens block 1 (16 .. 31) goes: the query at 47 sees from 32 on, that at 46 from 31.
    r = oracle_lib.tables_step([30, 46], [3, 3], [[5, 6, -1, -1], [7, 8, 9, -1]], [11, 12, 13, 14], [2, 4], 16, 4, 8)
    assert r["tables"].tolist() == [[5, 6, 13, -1], [7, 8, 9, 14]]
    assert r["slots"].tolist() == [6 * 16 + 14, 6 * 16 + 15, 13 * 16, 9 * 16 + 14, 9 * 16 + 15, 14 * 16, -1, -1]
    assert r["cu"].tolist() == [0, 3, 6] and r["next"].tolist() == [33, 49]
    assert r["counts"].tolist() == [4, 5] and r["ring"].tolist() == [8, 12, 13, 14]
