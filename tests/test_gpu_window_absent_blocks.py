"""Windowed attention over tables with ids outside the pool among the blocks that a call reads: they are
flagged, and their keys left out."""
import numpy as np
import pytest
import torch

from paper_2606_22983_amd import workloads as W
from tests.gpu_util import i32_dev
from tests.test_gpu_window_decode import Case as Decode
from tests.test_gpu_window_prefill import Case as Prefill
from tests.window_util import assert_within, visible

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    from paper_2606_22983_amd import kv as kv_mod
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return kv_mod


def attend_without(c, work, absent, rows, who, pos):
    """softmax(scale q K^T) V in 64 bits over the keys that a row sees, but for those of absent (session, block) pairs;
    also sum w |v| and the largest scale sum |q k|, as the oracle gives them."""
    hq, d = c.q.shape[1], c.d
    hkv = work.shape[3]
    nb = work.shape[1]
    kt = W.from_bf16(work[c.layer, :, 0]).reshape(nb, hkv, d // 8, 16, 8)
    vt = W.from_bf16(work[c.layer, :, 1]).reshape(nb, hkv, d, 16)
    out, mass = np.empty((len(rows), hq, d)), np.empty((len(rows), hq, d))
    score = np.empty((len(rows), hq))
    for i, r in enumerate(rows):
        s, p = int(who[r]), int(pos[r])
        t = np.arange(p + 1)
        t = t[visible(p, t, c.window, c.sinks)]
        t = t[[(s, b) not in absent for b in (t // 16).tolist()]]
        b, o = c.ses.tables[s, t // 16], t % 16
        k = kt[b, :, :, o].reshape(len(t), hkv, d).astype(np.float64)
        v = vt[b, :, :, o].astype(np.float64)
        q = W.from_bf16(c.q[r]).astype(np.float64)
        for h in range(hq):
            g = h // (hq // hkv)
            x = c.scale * (k[:, g] @ q[h])
            w = np.exp(x - x.max())
            w /= w.sum()
            out[i, h], mass[i, h] = w @ v[:, g], w @ np.abs(v[:, g])
            score[i, h] = (c.scale * (np.abs(k[:, g]) @ np.abs(q[h]))).max()
    return out, mass, score


def appended(c):
    work = c.ses.pool.copy()
    if c.kn is not None:
        c.oracle.append(work, 16, c.d, c.layer, c.ses.tables, c.who, c.pos, c.kn, c.vn)
    return work


def drop(c, absent):
    """Ids outside the pool for some blocks."""
    t = c.ses.tables.copy()
    for i, (s, b) in enumerate(sorted(absent)):
        t[s, b] = (-1, c.ses.pool.shape[1], 2**31 - 1, -2**31)[i % 4]
    c.tables.copy_(i32_dev(t))


# (turns, window, sinks, absent blocks): the first tokens' block, inside the window, its first and last
# block, one that only some rows see, the turn's own, one past the 512 blocks that a workgroup has threads for
PREFILL = [([(20, 100), (30, 50)], 64, 4, {(0, 6)}), ([(40, 700)], 300, 20, {(0, 0)}), ([(40, 700)], 300, 20, {(0, 1), (0, 40)}),
           ([(100, 400), (300, 900)], 200, 0, {(0, 13), (1, 60), (1, 70)}), ([(70, 33)], 1 << 29, 0, {(0, 2), (0, 5)}),
           ([(33, 9000)], 1 << 29, 0, {(0, 530)}), ([(301, 4000)], 2048, 4, {(0, 130), (0, 200), (0, 255)}), ([(40, 3)], 4, 300, {(0, 0)})]


@pytest.mark.parametrize("turns,window,sinks,absent", PREFILL)
@pytest.mark.parametrize("hq,hkv,d,append", [(8, 1, 128, False), (4, 2, 64, True), (16, 2, 64, False), (2, 2, 128, True)])
def test_prefill(kv, oracle_lib, turns, window, sinks, absent, hq, hkv, d, append):
    c = Prefill(kv, oracle_lib, turns, window, sinks, hq, hkv, d, append, seed=window % 999 + hq)
    work = appended(c)
    # rows that are left with a key
    left = [any((int(c.who[r]), int(b)) not in absent for b in np.unique(t[visible(c.pos[r], t, window, sinks)] // 16))
            for r in range(len(c.pos)) for t in [np.arange(c.pos[r] + 1)]]
    rows = np.nonzero(left)[0]
    rows = np.unique(np.concatenate([rows[:30], rows[-30:], np.random.default_rng(1).choice(rows, 30)]))
    ref = attend_without(c, work, absent, rows, c.who, c.pos)
    whole = np.arange(len(c.pos))
    other = whole[~np.isin(c.who, [s for s, _ in absent])]
    drop(c, absent)
    for mode in ("device", "host", "counters", "full"):
        c.data.copy_(torch.from_numpy(c.ses.pool.view(np.int16)).cuda().view(torch.bfloat16))
        out = c.run(mode)
        assert kv.ls_device_errors() == kv.LS_DEVERR_BLOCK_ID, mode
        assert_within(out[torch.from_numpy(rows).cuda()], *ref, d, "absent blocks, " + mode)
        if len(other):
            _, plain = c.reference(other)
            assert_within(out[torch.from_numpy(other).cuda()], *plain, d, "the other session, " + mode)


@pytest.mark.parametrize("lens,window,sinks,absent", [
    ([300, 100], 64, 4, {(0, 17)}), ([300, 100], 64, 4, {(0, 0), (1, 3)}), ([3000, 2500, 40], 1024, 20, {(0, 150), (0, 186), (1, 1)})])
@pytest.mark.parametrize("hq,hkv,d,append", [(8, 1, 128, False), (4, 2, 64, True)])
def test_decode(kv, oracle_lib, lens, window, sinks, absent, hq, hkv, d, append):
    c = Decode(kv, oracle_lib, lens, window, sinks, hq, hkv, d, append, seed=window)
    c.who = np.arange(len(lens))
    work = appended(c)
    ref = attend_without(c, work, absent, np.arange(len(lens)), c.who, c.pos)
    drop(c, absent)
    for host in (False, True):
        out = c.run(host)
        assert kv.ls_device_errors() == kv.LS_DEVERR_BLOCK_ID
        assert_within(out, *ref, d, "absent blocks, host lengths %s" % host)
