"""Accumulated attention weights, of decode steps and of turns, against sums of 64-bit probabilities."""
import numpy as np
import pytest
import torch

from paper_2606_22983_amd import workloads as W
from tests.cache_util import BLOCK, Cache, add_weights, assert_entries, attend, decode_reference, weight_bound
from tests.gpu_util import bf16_dev, i32_dev
from tests.window_util import assert_within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    from paper_2606_22983_amd import kv as kv_mod
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    kv_mod.ls_device_errors()
    return kv_mod


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def decode_check(kv, c, hq, what, layer=0, new=1, first=0, begin="apart", flags=0, seed=3, poison=True):
    rng = np.random.default_rng(seed)
    s, d, g = len(c.lens), c.d, hq // c.hkv
    q = W.normal_bf16(rng, (s, hq, d))
    w0, p0 = c.entries(rng)
    if poison:
        for i, n in enumerate(c.lens):                   # entries of new tokens and of slots without one mean nothing
            t = np.arange(max(0, n - new), -(-n // BLOCK) * BLOCK)
            w0[:, c.tables[i, t // BLOCK], :, t % BLOCK] = np.nan
    weights, positions = dev(w0), dev(p0)
    reused = np.maximum(c.lens - new, 0) if new is not None else None
    firsts = np.full(s, first) if np.isscalar(first) else np.asarray(first)
    begins = None if begin is None else rng.integers(0, 1 << 30, s)
    starts, members, prefix = c.group_arrays()
    pool = c.device(kv)
    n = kv.decode_weights_workspace_bytes(pool, s, hq, 0 if prefix is None else len(prefix),
                                          0 if members is None else len(members))
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    out = torch.full((s, hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    kv.paged_attn_decode_weights(pool, layer, bf16_dev(q), c.dtables, i32_dev(c.lens), d ** -0.5, out, weights,
                                 None if reused is None else positions, ws,
                                 reused_lens=None if reused is None else i32_dev(reused),
                                 first_positions=None if begins is None or reused is None else i32_dev(begins),
                                 first_lens=i32_dev(firsts) if firsts.any() else None, group_starts=starts,
                                 group_members=members, prefix_blocks=prefix)
    assert kv.ls_device_errors() == flags, what
    ref, mass, score, ps = decode_reference(c, layer, q, d ** -0.5)
    assert_within(out, ref, mass, score, d, what)
    w, pos, tol = w0.astype(np.float64), p0.copy(), np.zeros(w0.shape)
    for i, n in enumerate(c.lens):
        sums = ps[i].reshape(c.hkv, g, n).sum(1)
        each = np.stack([weight_bound(ps[i].reshape(c.hkv, 1, g, n)[h], score[i].reshape(c.hkv, 1, g)[h], d)
                         for h in range(c.hkv)])
        lo = max(int(firsts[i]), c.prefix_of(i))
        old = n if reused is None else int(reused[i])
        add_weights(c, layer, i, sums, each, w, pos, tol, lo, old, old if begins is None else int(begins[i]))
    same = np.isnan(w0) & (tol == 0)
    assert np.isnan(weights.cpu().numpy()[same]).all(), what
    assert_entries(torch.nan_to_num(weights), np.where(same, 0, w), tol, what)
    assert np.array_equal(positions.cpu().numpy(), pos), what


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("hkv,g", [(1, 1), (2, 2), (3, 4), (4, 8), (8, 1)])
@pytest.mark.parametrize("lens", [[1], [15, 16, 17, 0, 33], [2000, 1, 300]])
def test_decode(kv, d, hkv, g, lens):
    decode_check(kv, Cache(np.random.default_rng(1), lens, hkv, d, layers=2), hkv * g, "%s" % lens, layer=1)


@pytest.mark.parametrize("new,first,begin", [(None, 0, None), (0, 4, "apart"), (1, 37, None), (3, 16, "apart"), (40, 5, "apart"),
                                             (1, 1000, None)])
def test_decode_new_and_first_keys(kv, new, first, begin):
    c = Cache(np.random.default_rng(2), [100, 33, 1, 500, 40], 2, 128)
    decode_check(kv, c, 8, "new %s first %d" % (new, first), new=new, first=first, begin=begin, poison=new is not None)


def test_decode_groups(kv):
    rng = np.random.default_rng(4)
    lens = rng.integers(1, 300, 30)
    groups = [(list(range(0, 20, 2)), 9), ([1, 5, 3], 4), ([29], 2)]
    for m, p in groups:
        lens[m] += p * BLOCK
    lens[[2, 5]] = [70, 64]                              # inside their prefix, and at its end
    c = Cache(rng, lens, 2, 128, groups)
    decode_check(kv, c, 16, "groups", first=np.where(np.arange(30) == 8, 200, 0))


def test_decode_one_long_session_and_large_scores(kv):
    decode_check(kv, Cache(np.random.default_rng(5), [30000], 1, 128, key_scale=4.0), 8, "30000 keys")
    decode_check(kv, Cache(np.random.default_rng(6), [9000, 12, 7000], 4, 64, key_scale=0.1), 4, "flat scores")


def test_decode_accumulates_over_replays(kv):
    """Weights of a captured call grow by the same sums with every replay."""
    rng = np.random.default_rng(7)
    c = Cache(rng, [300, 20, 77], 2, 64)
    pool = c.device(kv)
    w0, p0 = c.entries(rng)
    q, lens = bf16_dev(W.normal_bf16(rng, (3, 8, 64))), i32_dev(c.lens)
    out = torch.empty_like(q)
    ws = torch.empty(kv.decode_weights_workspace_bytes(pool, 3, 8), dtype=torch.uint8, device="cuda")
    w = torch.zeros_like(dev(w0))
    kv.paged_attn_decode_weights(pool, 0, q, c.dtables, lens, 0.125, out, w, None, ws)
    once = w.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kv.paged_attn_decode_weights(pool, 0, q, c.dtables, lens, 0.125, out, w, None, ws)
    for i in range(2, 6):
        graph.replay()
        torch.cuda.synchronize()
        # (each addition rounds once)
        assert ((w - i * once).abs() <= i * i * 2.0 ** -24 * once).all()
    assert kv.ls_device_errors() == 0
    total = w.double().sum().item() / 5                  # every query gives 1 in all
    assert abs(total - 3 * 8) < 3 * 8 * 2.0 ** -12


def turn_check(kv, c, n, rows, hq, what, layer=0, first=0, begin="apart", seed=3, max_new=None):
    """The last n[s] tokens of every session are the turn."""
    rng = np.random.default_rng(seed)
    s, d, g = len(c.lens), c.d, hq // c.hkv
    n = np.asarray(n)
    ctx = c.lens - n
    cu = np.concatenate([[0], np.cumsum(n)])
    total = int(cu[-1])
    q = W.normal_bf16(rng, (total, hq, d))
    w0, p0 = c.entries(rng)
    for i in range(s):
        t = np.arange(ctx[i], -(-c.lens[i] // BLOCK) * BLOCK)
        w0[:, c.tables[i, t // BLOCK], :, t % BLOCK] = np.nan
    weights, positions = dev(w0), dev(p0)
    begins = None if begin is None else rng.integers(0, 1 << 30, s)
    firsts = np.full(s, first)
    pool = c.device(kv)
    longest = int(n.max()) if max_new is None else max_new
    size = kv.weights_prefill_workspace_bytes(pool, s, hq, total, longest, rows, c.tables.shape[1])
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    kv.kv_weights_prefill(pool, layer, bf16_dev(q), i32_dev(cu), i32_dev(ctx), longest, c.dtables, rows, d ** -0.5, weights,
                          positions, ws, first_positions=None if begins is None else i32_dev(begins),
                          first_lens=i32_dev(firsts) if first else None)
    assert kv.ls_device_errors() == 0, what
    w, pos, tol = w0.astype(np.float64), p0.copy(), np.zeros(w0.shape)
    for i in range(s):
        if not n[i]:
            continue
        k, v = c.rows(layer, i, np.arange(c.lens[i]))
        j = np.arange(max(0, n[i] - rows), n[i])
        seen = np.arange(c.lens[i])[None] <= (ctx[i] + j)[:, None]
        _, _, score, p = attend(W.from_bf16(q[cu[i] + j]).astype(np.float64), k, v, seen, d ** -0.5)
        p, score = p.reshape(len(j), c.hkv, g, -1), score.reshape(len(j), c.hkv, g)
        sums = p.sum((0, 2))
        each = np.stack([weight_bound(p[:, h], score[:, h], d) for h in range(c.hkv)])
        add_weights(c, layer, i, sums, each, w, pos, tol, first, int(ctx[i]), int(ctx[i] if begins is None else begins[i]))
        # a sum over rows in fp32, in an order of its own, and keys that no observed row sees (set to 0)
        t = np.arange(first, c.lens[i])
        tol[layer, c.tables[i, t // BLOCK], :, t % BLOCK] += 2.0 ** -12 * np.abs(w[layer, c.tables[i, t // BLOCK], :, t % BLOCK]) + 1e-30
    same = np.isnan(w0) & (tol == 0)
    assert np.isnan(weights.cpu().numpy()[same]).all(), what
    assert_entries(torch.nan_to_num(weights), np.where(same, 0, w), tol, what)
    assert np.array_equal(positions.cpu().numpy(), pos), what


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("hkv,g", [(1, 1), (2, 2), (3, 4), (4, 8)])
@pytest.mark.parametrize("rows", [1, 7, 64, 1000])
def test_turn(kv, d, hkv, g, rows):
    c = Cache(np.random.default_rng(1), [1, 40, 300, 77, 16], hkv, d, layers=2)
    turn_check(kv, c, [1, 40, 90, 0, 5], rows, hkv * g, "rows %d" % rows, layer=1)


@pytest.mark.parametrize("first,begin", [(0, None), (4, "apart"), (37, None), (2000, "apart")])
def test_turn_first_keys(kv, first, begin):
    c = Cache(np.random.default_rng(2), [60, 500], 2, 128)
    turn_check(kv, c, [20, 33], 16, 8, "first %d" % first, first=first, begin=begin)


def test_turn_of_many_rows(kv):
    """More rows than a round takes: 300 tokens of 8 heads."""
    turn_check(kv, Cache(np.random.default_rng(3), [450, 301], 2, 128), [300, 301], 400, 16, "many rows")
    turn_check(kv, Cache(np.random.default_rng(4), [1300], 1, 64), [1300], 1300, 2, "1300 tokens")


def test_turns_over_long_contexts(kv):
    """Chunks of every size: few and many keys, one session and many."""
    rng = np.random.default_rng(5)
    turn_check(kv, Cache(rng, [9000], 1, 128), [40], 32, 8, "one session")
    turn_check(kv, Cache(rng, [3000] * 9, 4, 64), [17] * 9, 16, 8, "nine sessions")
    lens = rng.integers(300, 900, 60)
    turn_check(kv, Cache(rng, lens, 8, 64), rng.integers(1, 30, 60), 4, 8, "sixty sessions", max_new=200)
    turn_check(kv, Cache(rng, [4000] * 40, 2, 64, key_scale=3.0), [3] * 40, 3, 2, "forty sessions")


def test_turns_that_cannot_be(kv):
    """Left out and flagged; the others are served."""
    rng = np.random.default_rng(6)
    c = Cache(rng, [64, 64, 64, 64], 1, 64, extra_cols=0)
    pool = c.device(kv)
    q = bf16_dev(W.normal_bf16(rng, (40, 2, 64)))
    for cu, ctx, max_new in (([0, 5, 3, 10, 20], [5, 5, 5, 5], 20), ([0, 30, 35, 40, 40], [5, 5, 5, 0], 20),
                             ([0, 5, 10, 20, 60], [5, 5, 5, 0], 40), ([0, 5, 10, 20, 30], [60, 5, -1, 5], 20),
                             ([-5, 5, 10, 20, 30], [5, 5, 5, 5], 20)):
        w, pos = torch.zeros((1, c.pool.shape[1], 1, BLOCK), device="cuda"), torch.zeros((1, c.pool.shape[1], 1, BLOCK), dtype=torch.int32, device="cuda")
        ws = torch.full((kv.weights_prefill_workspace_bytes(pool, 4, 2, 40, max_new, 8, 4),), 255, dtype=torch.uint8, device="cuda")
        kv.kv_weights_prefill(pool, 0, q, i32_dev(cu), i32_dev(ctx), max_new, c.dtables, 8, 0.125, w, pos, ws)
        assert kv.ls_device_errors() == kv.LS_DEVERR_LENGTH
        for s in range(4):
            n = cu[s + 1] - cu[s]
            fine = cu[s] >= 0 and 0 <= n <= max_new and cu[s + 1] <= 40 and 0 <= ctx[s] <= 64 - n
            got = w[0, c.dtables[s].long()].double().sum().item()
            want = min(n, 8) * 2 if fine else 0
            assert abs(got - want) <= 2.0 ** -12 * want, (cu, ctx, s)


def test_absent_blocks_get_no_weight(kv):
    rng = np.random.default_rng(8)
    c = Cache(rng, [100, 90], 2, 128)
    q = W.normal_bf16(rng, (2, 16, 128))
    qt = W.normal_bf16(rng, (40, 16, 128))
    c.tables[0, 3], c.tables[1, 0] = c.pool.shape[1], -1
    pool = c.device(kv)
    shape = (1, c.pool.shape[1], 2, BLOCK)
    w, pos = torch.zeros(shape, device="cuda"), torch.zeros(shape, dtype=torch.int32, device="cuda")
    ws = torch.full((kv.decode_weights_workspace_bytes(pool, 2, 16),), 255, dtype=torch.uint8, device="cuda")
    out = torch.empty((2, 16, 128), dtype=torch.bfloat16, device="cuda")
    kv.paged_attn_decode_weights(pool, 0, bf16_dev(q), c.dtables, i32_dev(c.lens), 128 ** -0.5, out, w, None, ws)
    assert kv.ls_device_errors() == kv.LS_DEVERR_BLOCK_ID
    assert abs(w.double().sum().item() - 2 * 16) < 2 * 16 * 2.0 ** -12 and out.isfinite().all()
    w.zero_()
    ws = torch.full((kv.weights_prefill_workspace_bytes(pool, 2, 16, 40, 20, 8, c.tables.shape[1]),), 255, dtype=torch.uint8, device="cuda")
    kv.kv_weights_prefill(pool, 0, bf16_dev(qt), i32_dev([0, 20, 40]), i32_dev(c.lens - 20), 20, c.dtables, 8, 128 ** -0.5, w,
                          pos, ws)
    assert kv.ls_device_errors() == kv.LS_DEVERR_BLOCK_ID
    assert abs(w.double().sum().item() - 2 * 8 * 16) < 2 * 8 * 16 * 2.0 ** -12
