"""Kernel variants of accumulated weights and eviction that batch and table sizes choose (on 256 CUs), and the forms in which
arguments are left out."""
import numpy as np
import pytest
import torch

from paper_2606_22983_amd import workloads as W
from tests.cache_util import BLOCK, Cache
from tests.gpu_util import bf16_dev, i32_dev
from tests.test_gpu_evict import check as evict_check
from tests.test_gpu_weights import decode_check, turn_check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    from paper_2606_22983_amd import kv as kv_mod
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    kv_mod.ls_device_errors()
    return kv_mod


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("sessions,hkv,length,n,rows,g", [
    (9, 4, 3000, 17, 16, 2),                             # two blocks a wave
    (40, 2, 4000, 3, 3, 1), (20, 8, 900, 70, 64, 4)])    # four, of few rows and of several stages
def test_turns_of_many_pairs(kv, d, sessions, hkv, length, n, rows, g):
    rng = np.random.default_rng(sessions)
    lens = length - rng.integers(0, 60, sessions)
    turn_check(kv, Cache(rng, lens, hkv, d), [n] * sessions, rows, hkv * g, "%d sessions of %d" % (sessions, length), first=4)


@pytest.mark.parametrize("sessions,ctx,n", [(1, 1700, 40), (4, 0, 90)])
def test_turns_in_wide_tables(kv, sessions, ctx, n):
    """Chunks of a table that no session fills."""
    c = Cache(np.random.default_rng(3), [ctx + n + 7 * i for i in range(sessions)], 2, 128, extra_cols=1500)
    turn_check(kv, c, [n] * sessions, 32, 8, "%d sessions in wide tables" % sessions)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("sessions", [512, 513, 1000, 2048])
def test_decode_weights_of_many_sessions(kv, d, sessions):
    """On either side of what the smaller schedule holds; groups of one tile and more, and sessions of none."""
    rng = np.random.default_rng(sessions)
    lens = rng.integers(1, 40, sessions)
    order = rng.permutation(sessions).tolist()
    groups = []
    for size, p in ((1, 3), (7, 2), (40, 5), (200, 1)):
        m = [order.pop() for _ in range(size)]
        lens[m] += p * BLOCK
        groups.append((m, p))
    lens[groups[2][0][:2]] = [3, 50]                     # shorter than their prefix
    lens[order[:5]] = 0
    decode_check(kv, Cache(rng, lens, 1, d, groups), 4, "%d sessions" % sessions)


@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("n,budget", [(2560, 1000), (2561, 1000), (9000, 700), (16384, 16000), (20000, 5000), (20000, 19990)])
def test_long_sessions_are_cut(kv, n, budget, apart):
    """Keys in LDS or not, moves of one workgroup or shared by several."""
    evict_check(kv, Cache(np.random.default_rng(8), [n, 17], 1, 128, extra_cols=0), budget, budget, budget // 3,
                "%d tokens to %d" % (n, budget), apart=apart)


@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_short_sessions_in_wide_tables_are_cut(kv, d, apart):
    c = Cache(np.random.default_rng(9), [300, 40, 101, 116, 0], 2, d, extra_cols=1024)
    evict_check(kv, c, 100, 110, 30, "wide table", apart=apart, first=[0, 4, 37, 16, 0])


@pytest.mark.parametrize("in_place", [False, True])
def test_no_sessions(kv, in_place):
    """The counters are written all the same."""
    c = Cache(np.random.default_rng(1), [20], 1, 64)
    pool = c.device(kv)
    i32 = dict(dtype=torch.int32, device="cuda")
    shape = (1, c.pool.shape[1], 1, BLOCK)
    weights, positions, none = torch.zeros(shape, device="cuda"), torch.zeros(shape, **i32), torch.empty(0, **i32)
    ring = torch.arange(9, **i32)
    counts = torch.tensor([(1 << 33) + 2, (1 << 33) + 7], device="cuda")
    after = counts if in_place else torch.full((2,), -1, device="cuda")
    kv.kv_evict(pool, none, torch.empty((0, 3), **i32), 5, 6, 1, none, weights, positions, torch.empty(0, **i32), free_ring=ring,
                free_counts=counts, next_counts=after)
    assert kv.ls_device_errors() == 0
    assert after.tolist() == [(1 << 33) + 2, (1 << 33) + 7] and ring.tolist() == list(range(9))
    assert not weights.any() and not positions.any()


def test_what_may_be_left_out(kv):
    """No groups, no first lengths, no first positions, no new keys: what the given arrays of that meaning give."""
    rng = np.random.default_rng(2)
    c = Cache(rng, [100, 37, 64], 2, 64)
    pool = c.device(kv)
    q, lens, reused = bf16_dev(W.normal_bf16(rng, (3, 8, 64))), i32_dev(c.lens), i32_dev(c.lens - 5)
    w0, p0 = (torch.from_numpy(x).cuda() for x in c.entries(rng))
    ws = torch.empty(kv.decode_weights_workspace_bytes(pool, 3, 8, 3, 3), dtype=torch.uint8, device="cuda")

    def call(**kw):
        w, p, out = w0.clone(), p0.clone(), torch.empty_like(q)
        kv.paged_attn_decode_weights(pool, 0, q, c.dtables, lens, 0.125, out, w, p if kw.get("reused_lens") is not None else None, ws, **kw)
        assert kv.ls_device_errors() == 0
        return out, w, p
    zeros, alone = i32_dev([0, 0, 0]), dict(group_starts=i32_dev([0, 1, 2, 3]), group_members=i32_dev([0, 1, 2]),
                                            prefix_blocks=i32_dev([0, 0, 0]))
    for short, whole in ((dict(reused_lens=reused), dict(reused_lens=reused, first_positions=reused, first_lens=zeros, **alone)),
                         (dict(), dict(reused_lens=lens, first_lens=zeros, **alone))):
        for a, b in zip(call(**short), call(**whole)):
            assert torch.equal(a, b)
    out, n = torch.empty_like(q), kv.decode_shared_workspace_bytes(pool, 3, 8, 0, 0)
    kv.paged_attn_decode_shared(pool, 0, q, c.dtables, lens, None, None, None, 0.125, out, ws[:n])
    assert kv.ls_device_errors() == 0 and torch.equal(out, call()[0])
