"""Accumulated weights of scores of every size: the keys of a session are equal, or of two kinds, so that the probabilities are
known whatever the scores, and scores of equal keys are the same bits."""
import numpy as np
import pytest
import torch

from paper_2606_22983_amd import workloads as W
from tests.cache_util import BLOCK, Cache
from tests.gpu_util import bf16_dev, i32_dev

pytestmark = pytest.mark.gpu

D, HKV, G = 64, 2, 2


@pytest.fixture(scope="module")
def kv():
    from paper_2606_22983_amd import kv as kv_mod
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    kv_mod.ls_device_errors()
    return kv_mod


def equal_keys(rng, lens, two):
    """Every K is a row of ones, or (two) that of every other key, and of the first, a little smaller."""
    c = Cache(rng, lens, HKV, D)
    for s, n in enumerate(lens):
        t = np.arange(n)
        k = np.ones((n, HKV, D), dtype=np.float32)
        if two:
            k[t % 2 == 0] = 1 - 2.0 ** -7
        c.write(0, s, t, W.to_bf16(k), W.normal_bf16(rng, (n, HKV, D)))
    return c


def probabilities(pos, n, two, positive):
    """Of keys 0 .. n - 1 for a row at position pos whose scores are far apart for the two kinds, or all zero (positive None)."""
    t = np.arange(n)
    p = t <= pos
    if two and positive is not None:
        best = p & (t % 2 == (1 if positive else 0))
        p = best if best.any() else p
    return p / p.sum()


# 2^-12 of each weight: exponential, division and fp32 sums, as everywhere.  Scores of equal keys have equal
# errors, which cancel; of two kinds at these sizes they are 2^7 or more apart, and the smaller one's probability is 0.
REL = 2.0 ** -12


@pytest.mark.parametrize("two", [False, True])
@pytest.mark.parametrize("size", [2.0 ** 14, 2.0 ** 22, -(2.0 ** 22), 2.0 ** 27, 2.0 ** 30, 2.0 ** 31, -(2.0 ** 31), 2.0 ** 34,
                                  -(2.0 ** 34), 2.0 ** 90, 0.0])
@pytest.mark.parametrize("sessions,ctx,n", [(1, 0, 100), (3, 333, 40), (40, 200, 6)])
def test_turn(kv, size, two, sessions, ctx, n):
    rng = np.random.default_rng(1)
    c = equal_keys(rng, [ctx + n] * sessions, two)
    q = W.to_bf16(np.full((sessions * n, HKV * G, D), size / 8, dtype=np.float32))       # score: 64 / 8 of it
    pool = c.device(kv)
    shape = (1, c.pool.shape[1], HKV, BLOCK)
    w, pos = torch.zeros(shape, device="cuda"), torch.zeros(shape, dtype=torch.int32, device="cuda")
    ws = torch.empty(kv.weights_prefill_workspace_bytes(pool, sessions, HKV * G, sessions * n, n, n, c.tables.shape[1]),
                     dtype=torch.uint8, device="cuda")
    kv.kv_weights_prefill(pool, 0, bf16_dev(q), i32_dev(np.arange(sessions + 1) * n), i32_dev([ctx] * sessions), n, c.dtables, n,
                          0.125, w, pos, ws)
    assert kv.ls_device_errors() == 0
    ref = G * sum(probabilities(ctx + j, ctx + n, two, size > 0 if size else None) for j in range(n))
    for s in range(sessions):
        t = np.arange(ctx + n)
        got = w.cpu().numpy()[0][c.tables[s, t // BLOCK], :, t % BLOCK].astype(np.float64)
        assert (np.abs(got - ref[:, None]) <= REL * ref[:, None]).all(), "worst %.3e" % np.nanmax(np.abs(got - ref[:, None]))


@pytest.mark.parametrize("two", [False, True])
@pytest.mark.parametrize("size", [2.0 ** 14, -(2.0 ** 22), 2.0 ** 34, 2.0 ** 90])
def test_decode(kv, size, two):
    rng = np.random.default_rng(2)
    lens = [1, 40, 700, 3000]
    c = equal_keys(rng, lens, two)
    q = W.to_bf16(np.full((4, HKV * G, D), size / 8, dtype=np.float32))
    pool = c.device(kv)
    w = torch.zeros((1, c.pool.shape[1], HKV, BLOCK), device="cuda")
    out = torch.empty((4, HKV * G, D), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(kv.decode_weights_workspace_bytes(pool, 4, HKV * G), dtype=torch.uint8, device="cuda")
    kv.paged_attn_decode_weights(pool, 0, bf16_dev(q), c.dtables, i32_dev(lens), 0.125, out, w, None, ws)
    assert kv.ls_device_errors() == 0
    for s, n in enumerate(lens):
        t = np.arange(n)
        ref = G * probabilities(n - 1, n, two, size > 0 if size else None)
        got = w.cpu().numpy()[0][c.tables[s, t // BLOCK], :, t % BLOCK].astype(np.float64)
        assert (np.abs(got - ref[:, None]) <= REL * ref[:, None]).all(), "worst %.3e" % np.nanmax(np.abs(got - ref[:, None]))
