"""Rows all of whose scores are far below zero: a softmax depends on their differences alone.  The keys are equal, so every
probability is one by their number, and the output the mean of V."""
import numpy as np
import pytest
import torch

from paper_2606_22983_amd import workloads as W
from tests.cache_util import BLOCK, Cache
from tests.gpu_util import bf16_dev, i32_dev

pytestmark = pytest.mark.gpu

HKV = 2


@pytest.fixture(scope="module")
def kv():
    from paper_2606_22983_amd import kv as kv_mod
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    kv_mod.ls_device_errors()
    return kv_mod


def cache(rng, lens, d, size, groups=()):
    """K rows of -sqrt(size), for q rows of sqrt(size): products of -d size."""
    c = Cache(rng, lens, HKV, d, groups)
    for s in sorted(range(len(lens)), key=lambda x: lens[x]):
        t = np.arange(lens[s])
        c.write(0, s, t, W.to_bf16(np.full((len(t), HKV, d), -size ** 0.5, dtype=np.float32)), W.normal_bf16(rng, (len(t), HKV, d)))
    return c


def assert_means(c, out, g, what):
    """P (equal ones, rounded to bf16 alike: nothing is lost), fp32 sums and division 2^-12 of the mean size, the output's own rounding."""
    got = out.float().cpu().numpy().astype(np.float64)
    for s, n in enumerate(c.lens):
        _, v = c.rows(0, s, np.arange(n))
        ref = np.repeat(v.mean(0), g, 0)
        tol = 2.0 ** -12 * np.repeat(np.abs(v).mean(0), g, 0) * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref)
        assert (np.abs(got[s] - ref) <= tol).all(), "%s: session %d" % (what, s)


SIZES = [2.0 ** 60, 2.0 ** 98, 2.0 ** 106, 2.0 ** 114]


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("d,g", [(128, 8), (64, 1)])
@pytest.mark.parametrize("members", [0, 2, 5, 20])               # no group; tiles of 16 rows, one, two; a tile of 128
def test_decode(kv, size, d, g, members):
    rng = np.random.default_rng(members)
    lens = np.array([1, 33, 300] + [700 + 11 * i for i in range(members)])
    c = cache(rng, lens, d, size, [(list(range(3, 3 + members)), 40)] if members else ())
    s = len(lens)
    pool, groups = c.device(kv), c.group_arrays()
    q = bf16_dev(W.to_bf16(np.full((s, HKV * g, d), size ** 0.5, dtype=np.float32)))
    out = torch.full((s, HKV * g, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    n = (1 if members else 0, members)
    ws = torch.full((kv.decode_shared_workspace_bytes(pool, s, HKV * g, *n),), 255, dtype=torch.uint8, device="cuda")
    kv.paged_attn_decode_shared(pool, 0, q, c.dtables, i32_dev(lens), *groups, d ** -0.5, out, ws)
    assert kv.ls_device_errors() == 0
    assert_means(c, out, g, "shared")
    w = torch.zeros((1, c.pool.shape[1], HKV, BLOCK), device="cuda")
    ws = torch.full((kv.decode_weights_workspace_bytes(pool, s, HKV * g, *n),), 255, dtype=torch.uint8, device="cuda")
    out.fill_(float("nan"))
    kv.paged_attn_decode_weights(pool, 0, q, c.dtables, i32_dev(lens), d ** -0.5, out, w, None, ws, group_starts=groups[0],
                                 group_members=groups[1], prefix_blocks=groups[2])
    assert kv.ls_device_errors() == 0
    assert_means(c, out, g, "weights")
    w = w.cpu().numpy()[0]
    for i, length in enumerate(lens):
        t = np.arange(c.prefix_of(i), length)
        assert (np.abs(w[c.tables[i, t // BLOCK], :, t % BLOCK] - g / length) <= 2.0 ** -12 * g / length).all()


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("d,g", [(128, 8), (64, 1)])
@pytest.mark.parametrize("sessions,ctx,n", [(1, 0, 70), (2, 500, 9), (30, 300, 5)])
def test_turn(kv, size, d, g, sessions, ctx, n):
    rng = np.random.default_rng(sessions)
    c = cache(rng, [ctx + n] * sessions, d, size)
    pool = c.device(kv)
    q = bf16_dev(W.to_bf16(np.full((sessions * n, HKV * g, d), size ** 0.5, dtype=np.float32)))
    shape = (1, c.pool.shape[1], HKV, BLOCK)
    w, pos = torch.zeros(shape, device="cuda"), torch.zeros(shape, dtype=torch.int32, device="cuda")
    ws = torch.full((kv.weights_prefill_workspace_bytes(pool, sessions, HKV * g, sessions * n, n, n, c.tables.shape[1]),), 255,
                    dtype=torch.uint8, device="cuda")
    kv.kv_weights_prefill(pool, 0, q, i32_dev(np.arange(sessions + 1) * n), i32_dev([ctx] * sessions), n, c.dtables, n, d ** -0.5, w,
                          pos, ws)
    assert kv.ls_device_errors() == 0
    t = np.arange(ctx + n)
    ref = sum((t <= ctx + j) * (g / (ctx + j + 1)) for j in range(n))
    for s in range(sessions):
        got = w.cpu().numpy()[0][c.tables[s, t // BLOCK], :, t % BLOCK]
        assert (np.abs(got - ref[:, None]) <= 2.0 ** -12 * ref[:, None]).all()
