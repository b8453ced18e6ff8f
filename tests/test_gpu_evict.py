"""Eviction by accumulated weight against a slot by slot one on the host: every bit is defined."""
import numpy as np
import pytest
import torch

from paper_2606_22983_amd import workloads as W
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


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def spread(c, rng, next_pos, ties=0):
    """Weights and positions: every session's tokens at distinct positions below its next one, in any order."""
    w, pos = c.entries(rng)
    if ties:
        w = rng.integers(0, ties, w.shape).astype(np.float32)
    for s, n in enumerate(c.lens):
        t = np.arange(n)
        for layer in range(c.layers):
            for h in range(c.hkv):
                pos[layer, c.tables[s, t // BLOCK], h, t % BLOCK] = rng.permutation(next_pos[s] - n + t)
    return w, pos


def ring_of(nb, held, start=(1 << 33) + 7):
    ring = np.full(2 * nb, -1, dtype=np.int32)
    free = np.setdiff1d(np.arange(nb), held)
    ring[(np.arange(len(free)) + start) % len(ring)] = free
    return ring, np.array([start, start + len(free)], dtype=np.int64)


def check(kv, c, budget, limit, recent, what, first=None, next_pos=None, w=None, pos=None, layers=None, apart=False, ring=True,
          ties=0, seed=3, in_place=False):
    rng = np.random.default_rng(seed)
    s = len(c.lens)
    firsts = np.zeros(s, dtype=np.int64) if first is None else np.asarray(first)
    next_pos = c.lens * 2 + 3 if next_pos is None else np.asarray(next_pos)
    if w is None:
        w, pos = spread(c, rng, next_pos, ties)
    lb, lc = layers or (0, c.layers)
    ref, wr, pr, keep = evict_reference(c.pool, c.tables, c.lens, budget, limit, recent, firsts, next_pos, w, pos,
                                        range(lb, lb + lc), c.d)
    pool = c.device(kv)
    weights, positions = dev(w), dev(pos)
    wn, pn = (torch.full_like(weights, 7.5), torch.full_like(positions, -77)) if apart else (None, None)
    nxt = torch.full((s,), -5, dtype=torch.int32, device="cuda")
    held = c.tables[(np.arange(c.tables.shape[1])[None] < -(-c.lens // BLOCK)[:, None])]
    hr, hc = ring_of(c.pool.shape[1], held)
    dring, dcounts, after = dev(hr), dev(hc), torch.empty(2, dtype=torch.int64, device="cuda")
    after = dcounts if in_place else after
    lens = i32_dev(c.lens)

    def call():
        kv.kv_evict(pool, lens, c.dtables, budget, limit, recent, i32_dev(next_pos), weights, positions, nxt, wn, pn,
                    None if first is None else i32_dev(firsts), lb, lc, *((dring, dcounts, after) if ring else ()))
    call()
    assert kv.ls_device_errors() == 0, what
    gone = [c.tables[i, j] for i in range(s) for j in range(-(-int(keep[i]) // BLOCK), -(-int(c.lens[i]) // BLOCK))]

    def compare():
        assert equal(bits(c.data).reshape(ref.shape), ref), what
        assert equal(nxt.cpu().numpy(), keep), what
        if apart:
            a, b = np.full_like(wr, 7.5), np.full_like(pr, -77)
            for i in range(s):
                t = np.arange(keep[i])
                at = (slice(lb, lb + lc), c.tables[i, t // BLOCK], slice(None), t % BLOCK)
                a[at], b[at] = wr[at], pr[at]
            assert equal(weights.cpu().numpy(), w) and equal(positions.cpu().numpy(), pos), what
            assert equal(wn.cpu().numpy(), a) and equal(pn.cpu().numpy(), b), what
        else:
            assert equal(weights.cpu().numpy(), wr) and equal(positions.cpu().numpy(), pr), what
        if ring:
            r = hr.copy()
            r[(hc[1] + np.arange(len(gone))) % len(r)] = gone
            assert equal(dring.cpu().numpy(), r) and after.tolist() == [hc[0], hc[1] + len(gone)], what
    compare()
    if apart:
        call()                                            # made again, with the same result
        assert kv.ls_device_errors() == 0, what
        compare()
    return pool


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("hkv", [1, 4])
@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("budget,limit,recent", [(64, 64, 0), (100, 115, 20), (33, 40, 33), (1, 1, 0), (200, 215, 150)])
def test_sizes(kv, d, hkv, apart, budget, limit, recent):
    lens = [1, 0, 64, 65, 101, 116, 215, 216, 300, 40]
    c = Cache(np.random.default_rng(1), lens, hkv, d, layers=2)
    check(kv, c, budget, limit, recent, "budget %d" % budget, apart=apart)


@pytest.mark.parametrize("first", [[0, 4, 16, 37, 100], [500, 300, 99, 101, 0]])
def test_first_slots(kv, first):
    """First tokens stay where they are, also where they are more than the budget, or than the session."""
    check(kv, Cache(np.random.default_rng(2), [150, 260, 99, 400, 120], 2, 64), 100, 110, 30, "first %s" % first, first=first)


@pytest.mark.parametrize("ties", [1, 2, 5])
def test_ties_go_to_the_lower_slot(kv, ties):
    check(kv, Cache(np.random.default_rng(3), [130, 500, 90], 2, 64), 80, 90, 10, "%d values" % ties, ties=ties)


def test_weights_of_every_kind(kv):
    """NaN ranks lowest, infinities and both zeros as numbers, denormals and negatives in their order."""
    c = Cache(np.random.default_rng(4), [200, 190], 2, 64)
    rng = np.random.default_rng(5)
    next_pos = c.lens * 2
    w, pos = spread(c, rng, next_pos)
    odd = np.array([np.nan, np.inf, -np.inf, 0.0, -0.0, 1e-42, -1e-42, 3.0, -3.0, 1e38], dtype=np.float32)
    w[:] = rng.choice(odd, w.shape)
    for budget in (30, 100, 150, 185):
        check(kv, c, budget, budget, 5, "odd weights, budget %d" % budget, next_pos=next_pos, w=w, pos=pos)
    check(kv, c, 100, 100, 0, "all NaN", next_pos=next_pos, w=np.full_like(w, np.nan), pos=pos)


def test_only_the_latest_are_left(kv):
    """Recent tokens fill the budget; none is recent; positions past what a next one says."""
    c = Cache(np.random.default_rng(6), [300, 50], 1, 128)
    rng = np.random.default_rng(7)
    w, pos = spread(c, rng, c.lens)
    check(kv, c, 40, 40, 40, "recent = budget", next_pos=c.lens, w=w, pos=pos)
    check(kv, c, 40, 40, 10, "none recent", next_pos=c.lens + 5000, w=w, pos=pos)
    check(kv, c, 40, 40, 10, "all recent", next_pos=[-2**31 + 3, 5], w=w, pos=pos)      # (more than there is room: lower slots)


@pytest.mark.parametrize("n,budget", [(2304, 2000), (2561, 1000), (4100, 2100), (9000, 700), (16384, 16000), (20000, 5000), (20000, 19990)])
def test_long_sessions(kv, n, budget):
    """Keys in LDS, and sessions longer than it holds; more moves than one batch takes."""
    check(kv, Cache(np.random.default_rng(8), [n, 17], 1, 64), budget, budget, budget // 3, "%d tokens to %d" % (n, budget))


def test_layers_of_a_range_and_no_ring(kv):
    c = Cache(np.random.default_rng(9), [100, 170], 3, 64, layers=4)
    check(kv, c, 60, 70, 20, "layers 1 and 2", layers=(1, 2), ring=False)
    check(kv, c, 60, 70, 20, "layer 3", layers=(3, 1))


def test_shared_blocks_stay(kv):
    """Sessions that share a prefix below their first lengths."""
    rng = np.random.default_rng(10)
    lens = 5 * BLOCK + np.array([60, 100, 3, 200])
    c = Cache(rng, lens, 2, 64, [([0, 1, 2, 3], 5)])
    w, pos = c.entries(rng)
    check(kv, c, 130, 140, 20, "shared", first=[80] * 4, w=w, pos=pos, apart=True)


def test_many_sessions(kv):
    rng = np.random.default_rng(11)
    lens = rng.integers(0, 60, 2500)
    c = Cache(rng, lens, 1, 64)
    check(kv, c, 30, 33, 8, "2500 sessions")


@pytest.mark.parametrize("n", [1023, 1024, 1025])
@pytest.mark.parametrize("in_place", [False, True])
def test_a_thousand_sessions(kv, n, in_place):
    """On both sides of what one launch plans and serves; counters that advance in place."""
    rng = np.random.default_rng(n)
    check(kv, Cache(rng, rng.integers(0, 50, n), 2, 64), 20, 24, 6, "%d sessions" % n, in_place=in_place)


@pytest.mark.parametrize("in_place", [False, True])
def test_refused_as_a_whole(kv, in_place):
    c = Cache(np.random.default_rng(12), [100, 70], 2, 64, extra_cols=0)
    rng = np.random.default_rng(13)
    w, pos = spread(c, rng, c.lens * 2)
    cap = c.tables.shape[1] * BLOCK
    for lens, counts, size, flag in (([100, -1], (0, 2), 50, kv.LS_DEVERR_LENGTH), ([cap + 1, 70], (0, 2), 50, kv.LS_DEVERR_LENGTH),
                                     ([100, 70], (0, 49), 50, kv.LS_DEVERR_FREE_LIST), ([100, 70], (5, 3), 50, kv.LS_DEVERR_FREE_LIST),
                                     ([100, 70], (-1, 3), 50, kv.LS_DEVERR_FREE_LIST), ([100, 70], (0, 51), 50, kv.LS_DEVERR_FREE_LIST)):
        pool = c.device(kv)
        weights, positions = dev(w), dev(pos)
        ring = torch.arange(size, dtype=torch.int32, device="cuda")
        before, after = torch.tensor(counts, device="cuda"), torch.empty(2, dtype=torch.int64, device="cuda")
        after = before if in_place else after
        nxt = torch.empty(2, dtype=torch.int32, device="cuda")
        kv.kv_evict(pool, i32_dev(lens), c.dtables, 20, 30, 5, i32_dev([300, 300]), weights, positions, nxt, free_ring=ring,
                    free_counts=before, next_counts=after)
        assert kv.ls_device_errors() == flag
        assert nxt.tolist() == lens and after.tolist() == list(counts) and ring.tolist() == list(range(size))
        assert equal(bits(c.data).reshape(c.pool.shape), c.pool)
        assert equal(weights.cpu().numpy(), w) and equal(positions.cpu().numpy(), pos)


def test_blocks_outside_the_pool(kv):
    """Their tokens rank lowest and are not moved; nothing else is written."""
    c = Cache(np.random.default_rng(14), [200], 1, 64, layers=2)
    rng = np.random.default_rng(15)
    w, pos = spread(c, rng, c.lens * 4)
    pos[:] = -5
    tables = c.tables.copy()
    for col in (2, 11):                                   # below the budget, and behind it
        c.tables = tables.copy()
        c.tables[0, col] = c.pool.shape[1] if col == 2 else -1
        pool = c.device(kv)
        weights, positions = dev(w), dev(pos)
        nxt = torch.empty(1, dtype=torch.int32, device="cuda")
        kv.kv_evict(pool, i32_dev([200]), c.dtables, 150, 150, 0, i32_dev([800]), weights, positions, nxt)
        assert kv.ls_device_errors() == kv.LS_DEVERR_BLOCK_ID and nxt.tolist() == [150]
        after = bits(c.data).reshape(c.pool.shape)
        used = tables[0, :13]
        other = np.setdiff1d(np.arange(c.pool.shape[1]), used[:10])
        assert equal(after[:, other], c.pool[:, other])       # blocks behind the budget are only read
        if col == 2:
            assert equal(after[:, tables[0, 2]], c.pool[:, tables[0, 2]])
    c.tables = tables


@pytest.mark.parametrize("in_place", [True, False])
def test_captured_and_replayed(kv, in_place):
    """Entries in place, counters that advance: every replay cuts what has grown since."""
    c = Cache(np.random.default_rng(16), [120, 90, 61], 2, 64)
    rng = np.random.default_rng(17)
    w, pos = spread(c, rng, c.lens * 2)
    pool = c.device(kv)
    weights, positions, lens, nxt = dev(w), dev(pos), i32_dev(c.lens), i32_dev([0, 0, 0])
    next_pos = i32_dev(c.lens * 2)
    ring, counts = (dev(x) for x in ring_of(c.pool.shape[1], np.arange(c.pool.shape[1])))

    after = counts if in_place else torch.empty_like(counts)

    def call():
        kv.kv_evict(pool, lens, c.dtables, 50, 60, 10, next_pos, weights, positions, nxt, free_ring=ring, free_counts=counts,
                    next_counts=after)
        if not in_place:
            counts.copy_(after)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call()
    for step in range(3):
        host = [bits(c.data).reshape(c.pool.shape), weights.cpu().numpy(), positions.cpu().numpy()]
        ref, wr, pr, keep = evict_reference(host[0], c.tables, lens.tolist(), 50, 60, 10, [0] * 3, next_pos.tolist(), host[1], host[2],
                                            [0], 64)
        given = int(counts[1])
        graph.replay()
        torch.cuda.synchronize()
        assert equal(bits(c.data).reshape(c.pool.shape), ref) and nxt.tolist() == keep.tolist()
        assert equal(weights.cpu().numpy(), wr) and equal(positions.cpu().numpy(), pr)
        assert int(counts[1]) - given == sum(-(-a // BLOCK) - -(-b // BLOCK) for a, b in zip(lens.tolist(), keep.tolist()))
        lens.copy_(nxt + torch.tensor([30, 7, 11], dtype=torch.int32, device="cuda"))
        next_pos.add_(30)
    assert kv.ls_device_errors() == 0
