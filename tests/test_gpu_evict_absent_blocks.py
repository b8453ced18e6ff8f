"""Eviction of sessions some of whose blocks are not in the pool: no token that stays is moved into one of these, or lost."""
import numpy as np
import pytest
import torch

from tests.cache_util import BLOCK, Cache, bits, evict_reference
from tests.gpu_util import i32_dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    from paper_2606_22983_amd import kv as kv_mod
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    kv_mod.ls_device_errors()
    return kv_mod


def equal(a, b):
    return bool(np.array_equal(a, b, equal_nan=a.dtype.kind == "f"))


@pytest.mark.parametrize("d,n,budget,recent", [(64, 300, 200, 60), (128, 200, 100, 100), (128, 120, 37, 5), (64, 20000, 9000, 300),
                                               (64, 2700, 1000, 1000)])
@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("kind", ["nan", "numbers"])
def test_every_bit(kv, d, n, budget, recent, apart, kind):
    """As if the slots of such blocks below the budget were kept tokens and those behind it the first to go."""
    rng = np.random.default_rng(n)
    c = Cache(rng, [n, 50], 2, d, layers=2)
    w, pos = c.entries(rng)
    t = np.arange(n)
    for layer in range(2):
        for h in range(2):
            pos[layer, c.tables[0, t // BLOCK], h, t % BLOCK] = rng.permutation(n) + 7
    if kind == "nan":
        w[rng.random(w.shape) < 0.9] = np.nan
    next_pos = [n + 7, 1000]
    last = -(-n // BLOCK) - 1
    absent = sorted({1, budget // BLOCK, (budget + n) // 2 // BLOCK, last})
    # the reference: weights that put these slots first and last
    ids = c.tables[0, absent].copy()
    wr, pr = w.copy(), pos.copy()
    for col, b in zip(absent, ids):
        for o in range(BLOCK):
            if col * BLOCK + o < budget:
                pr[:, b, :, o] = 1 << 30                  # (a latest token)
            else:
                wr[:, b, :, o], pr[:, b, :, o] = np.nan, -1
    at = np.zeros(n, dtype=bool)
    for col in absent:
        at[col * BLOCK:(col + 1) * BLOCK] = True
    behind = at & (t >= budget)
    if kind == "nan":
        # among NaN the reference evicts the highest slots: those of absent blocks have to be the first to go, so the
        # others behind them are lifted to numbers
        b, o = c.tables[0, t[~behind] // BLOCK], t[~behind] % BLOCK
        first_behind = t[behind].min()
        lift = t[~behind] >= first_behind
        for arr in (w, wr):
            x = arr[:, b[lift], :, o[lift]]
            arr[:, b[lift], :, o[lift]] = np.where(np.isnan(x), np.float32(0.25), x)
    ref_pool, ref_w, ref_p, keep = evict_reference(c.pool, c.tables, c.lens, budget, budget, recent, [0, 0], next_pos, wr, pr, range(2), d)
    for arr, old in ((ref_w, w), (ref_p, pos)):
        arr[:, ids] = old[:, ids]                         # (nothing is written there)
    tables = c.tables.copy()
    c.tables[0, absent] = [c.pool.shape[1], -1, 2**31 - 1, -7][:len(absent)]
    pool = c.device(kv)
    weights, positions = torch.from_numpy(w).cuda(), torch.from_numpy(pos).cuda()
    wn, pn = (torch.full_like(weights, 7.5), torch.full_like(positions, -77)) if apart else (None, None)
    nxt = torch.empty(2, dtype=torch.int32, device="cuda")
    kv.kv_evict(pool, i32_dev(c.lens), c.dtables, budget, budget, recent, i32_dev(next_pos), weights, positions, nxt, wn, pn)
    assert kv.ls_device_errors() == kv.LS_DEVERR_BLOCK_ID and nxt.tolist() == keep.tolist() == [budget, min(50, budget)]
    assert equal(bits(c.data).reshape(ref_pool.shape), ref_pool)
    if not apart:
        assert equal(weights.cpu().numpy(), ref_w) and equal(positions.cpu().numpy(), ref_p)
        return
    a, b = np.full_like(ref_w, 7.5), np.full_like(ref_p, -77)
    for s in range(2):
        x = np.arange(keep[s])
        x = x[~np.isin(x // BLOCK, absent)] if s == 0 else x
        i = (slice(None), tables[s, x // BLOCK], slice(None), x % BLOCK)
        a[i], b[i] = ref_w[i], ref_p[i]
    assert equal(wn.cpu().numpy(), a) and equal(pn.cpu().numpy(), b)
