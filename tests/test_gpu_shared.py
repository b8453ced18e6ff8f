"""Decode of sessions that share prefixes, against the 64-bit result over every session's own keys."""
import numpy as np
import pytest
import torch

from paper_2606_22983_amd import workloads as W
from tests.cache_util import BLOCK, Cache, decode_reference
from tests.gpu_util import bf16_dev, i32_dev
from tests.window_util import assert_within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    from paper_2606_22983_amd import kv as kv_mod
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    kv_mod.ls_device_errors()
    return kv_mod


def run(kv, c, pool, q, layer=0, groups=None, lens=None, stream=None, ws=None):
    s, hq, d = q.shape
    starts, members, prefix = c.group_arrays() if groups is None else groups
    if ws is None:
        n = kv.decode_shared_workspace_bytes(pool, s, hq, 0 if prefix is None else len(prefix),
                                             0 if members is None else len(members))
        assert n > 0
        ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")         # NaN wherever it is read before written
    out = torch.full((s, hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    kv.paged_attn_decode_shared(pool, layer, q, c.dtables, i32_dev(c.lens if lens is None else lens), starts, members, prefix,
                                d ** -0.5, out, ws, stream=stream)
    return out


def check(kv, c, hq, what, layer=0, flags=0, seed=7):
    rng = np.random.default_rng(seed)
    q = W.normal_bf16(rng, (len(c.lens), hq, c.d))
    pool = c.device(kv)
    dq = bf16_dev(q)
    out = run(kv, c, pool, dq, layer)
    assert kv.ls_device_errors() == flags, what
    ref, mass, score, _ = decode_reference(c, layer, q, c.d ** -0.5)
    assert_within(out, ref, mass, score, c.d, what)
    assert torch.equal(out, run(kv, c, pool, dq, layer)), what              # the same bits again
    return pool, dq, out


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("hkv,g", [(1, 1), (2, 2), (3, 4), (2, 8), (5, 1)])
@pytest.mark.parametrize("sizes", [(1,), (2, 3), (9, 1, 4)])
def test_groups(kv, d, hkv, g, sizes):
    rng = np.random.default_rng(hkv * 100 + g * 10 + len(sizes))
    n = sum(sizes) + 3                                    # three sessions in no group
    order = rng.permutation(n)
    cuts = np.cumsum((0,) + sizes)
    groups = [(order[a:b].tolist(), int(rng.integers(1, 12))) for a, b in zip(cuts, cuts[1:])]
    lens = rng.integers(1, 200, n)
    for m, p in groups:
        lens[m] += p * BLOCK
    check(kv, Cache(rng, lens, hkv, d, groups), hkv * g, "groups %s" % (sizes,))


@pytest.mark.parametrize("members", [1, 2, 4, 5, 8, 9, 17, 40])
@pytest.mark.parametrize("g", [8, 3 - 2])
def test_rows_of_a_group(kv, members, g):
    """Groups whose query rows fill one tile of 16, 32 or 64 rows, or run over into more."""
    rng = np.random.default_rng(members)
    p = 37
    lens = p * BLOCK + rng.integers(0, 40, members)
    check(kv, Cache(rng, lens, 2, 128, [(list(range(members)), p)]), 2 * g, "%d members" % members)


@pytest.mark.parametrize("lens,prefix", [
    ([1, 1], 0), ([16, 16], 1), ([17, 16, 0], 1), ([0, 0, 5], 0), ([160, 159, 145, 161], 10), ([160, 3, 0, 40, 161], 10),
    ([100, 90, 0], 20), ([0, 0], 3), ([1], 1), ([33, 12], 30), ([15, 16], 1),
])
def test_lengths_around_the_prefix(kv, lens, prefix):
    """Members at, before and behind the end of the prefix, with no key at all, prefixes longer than any member."""
    rng = np.random.default_rng(sum(lens))
    c = Cache(rng, lens, 2, 128, [(list(range(len(lens))), prefix)], extra_cols=35)
    _, _, out = check(kv, c, 16, "lens %s prefix %d" % (lens, prefix))
    for s, n in enumerate(lens):
        if n == 0:
            assert (out[s] == 0).all()


@pytest.mark.parametrize("members", [5, 12, 40])                # rows in a tile of 16, tiles of 16, a tile of 128
def test_keys_that_a_shorter_member_does_not_see(kv, members):
    """K and V that are not finite, in shared blocks behind a member's keys: its row does not know."""
    rng = np.random.default_rng(members)
    lens = np.full(members, 100)
    short = [1, 2, members - 1]
    lens[short] = [60, 0, 37]
    c = Cache(rng, lens, 2, 128, [(list(range(members)), 5)])
    pool, q, clean = check(kv, c, 8 if members == 5 else 16, "finite")
    for k, v in ((np.inf, 1.0), (1.0, np.inf), (np.nan, np.nan)):
        for t in (60, 79):
            row = np.ones((1, 2, 128))
            c.write(0, 0, np.array([t]), W.to_bf16((row * k).astype(np.float32)), W.to_bf16((row * v).astype(np.float32)))
        out = run(kv, c, c.device(kv), q)
        assert kv.ls_device_errors() == 0
        assert torch.equal(out[short], clean[short])
        assert not torch.isfinite(out[0]).all()


@pytest.mark.parametrize("lens", [[1], [2, 31, 32, 33], [5000], [20000, 1, 700], [0, 64, 0]])
@pytest.mark.parametrize("d,hkv,g", [(128, 4, 8), (64, 1, 1), (128, 8, 2)])
def test_without_groups(kv, lens, d, hkv, g):
    check(kv, Cache(np.random.default_rng(len(lens)), lens, hkv, d), hkv * g, "no groups %s" % lens)


def test_long_prefix_and_many_parts(kv):
    """A prefix that every workgroup has a part of, large scores among them, in the second layer of two."""
    rng = np.random.default_rng(5)
    lens = 600 * BLOCK + rng.integers(0, 300, 12)
    c = Cache(rng, lens, 2, 128, [(list(range(3, 12)), 600)], layers=2, key_scale=4.0)
    check(kv, c, 16, "long prefix", layer=1)


def test_many_sessions_and_groups(kv):
    rng = np.random.default_rng(6)
    n = 700
    order = rng.permutation(n).tolist()
    groups, lens = [], rng.integers(0, 30, n)
    while len(order) > 100:
        m = [order.pop() for _ in range(int(rng.integers(1, 5)))]
        p = int(rng.integers(0, 4))
        lens[m] += p * BLOCK
        groups.append((m, p))
    check(kv, Cache(rng, lens, 1, 64, groups), 2, "700 sessions in %d groups" % len(groups))


def test_at_the_limits(kv):
    """2048 sessions, all in groups; a table of 16384 blocks."""
    rng = np.random.default_rng(8)
    lens = rng.integers(1, 40, 2048)
    lens += 2 * BLOCK
    check(kv, Cache(rng, lens, 1, 64, [(list(range(i, 2048, 64)), 2) for i in range(64)]), 8, "2048 sessions")
    lens = [16384 * BLOCK, 16383 * BLOCK + 1]
    check(kv, Cache(rng, lens, 1, 64, [([0, 1], 16000)], extra_cols=0), 1, "16384 blocks")


def test_the_first_table_is_not_the_longest(kv):
    """The group's first member has sat out so long that its table row says nothing."""
    rng = np.random.default_rng(9)
    c = Cache(rng, [0, 70, 300, 290], 2, 64, [([0, 1, 3, 2], 18)])
    c.tables[0] = 2**31 - 1
    check(kv, c, 8, "stale first member")


@pytest.mark.parametrize("what", ["twice", "outside", "negative", "falling", "open start", "open end", "long prefix", "negative prefix"])
def test_groups_that_cannot_be(kv, what):
    """Flagged, and every session computed over its own table."""
    rng = np.random.default_rng(10)
    c = Cache(rng, [100, 200, 300, 50], 2, 128, [([0, 1], 3), ([2, 3], 2)])
    starts, members, prefix = [0, 2, 4], [0, 1, 2, 3], [3, 2]
    if what == "twice":
        members[3] = 1
    elif what == "outside":
        members[0] = 4
    elif what == "negative":
        members[2] = -1
    elif what == "falling":
        starts[1] = 5
    elif what == "open start":
        starts[0] = 1
    elif what == "open end":
        starts[2] = 3
    elif what == "long prefix":
        prefix[1] = c.tables.shape[1] + 1
    else:
        prefix[0] = -1
    pool = c.device(kv)
    q = W.normal_bf16(rng, (4, 16, 128))
    out = run(kv, c, pool, bf16_dev(q), groups=(i32_dev(starts), i32_dev(members), i32_dev(prefix)))
    assert kv.ls_device_errors() == kv.LS_DEVERR_GROUP
    assert_within(out, *decode_reference(c, 0, q, 128 ** -0.5)[:3], 128, what)


def test_lengths_out_of_range(kv):
    rng = np.random.default_rng(11)
    c = Cache(rng, [80, 64, 96], 1, 64, [([0, 2], 4)], extra_cols=0)
    pool = c.device(kv)
    q = W.normal_bf16(rng, (3, 4, 64))
    out = run(kv, c, pool, bf16_dev(q), lens=[80, -5, 2**31 - 1])
    assert kv.ls_device_errors() == kv.LS_DEVERR_LENGTH
    assert (out[1] == 0).all()
    ref, mass, score, _ = decode_reference(c, 0, q, 0.125)
    assert_within(out[[0, 2]], ref[[0, 2]], mass[[0, 2]], score[[0, 2]], 64, "other sessions")


def test_blocks_outside_the_pool(kv):
    """Keys of such a block are left out, in the prefix and behind it."""
    rng = np.random.default_rng(12)
    c = Cache(rng, [150, 170, 60], 2, 128, [([0, 1], 6)])
    q = W.normal_bf16(rng, (3, 16, 128))
    c.tables[1, 2] = c.pool.shape[1]                      # (the longest member's row is read)
    c.tables[0, 2] = -1
    c.tables[2, 1] = 2**31 - 1
    pool = c.device(kv)
    out = run(kv, c, pool, bf16_dev(q))
    assert kv.ls_device_errors() == kv.LS_DEVERR_BLOCK_ID
    ref = []
    from tests.cache_util import attend
    for s, hole in enumerate((2, 2, 1)):
        t = np.array([t for t in range(c.lens[s]) if t // BLOCK != hole])
        k, v = c.rows(0, s, t)
        ref.append([x[0] for x in attend(W.from_bf16(q[s:s + 1]).astype(np.float64), k, v, np.ones((1, len(t)), bool), 128 ** -0.5)[:3]])
    assert_within(out, *(np.stack(x) for x in zip(*ref)), 128, "without blocks")


def test_two_captured_calls_with_their_own_workspaces_and_lengths_that_grow(kv):
    rng = np.random.default_rng(13)
    c = Cache(rng, 8 * BLOCK + rng.integers(20, 200, 6), 2, 128, [([0, 2, 4], 8), ([5, 1], 7)])
    pool = c.device(kv)
    full, groups = c.lens.copy(), c.group_arrays()
    q = [bf16_dev(W.normal_bf16(rng, (6, 16, 128))) for _ in range(2)]
    lens = i32_dev(full)
    n = kv.decode_shared_workspace_bytes(pool, 6, 16, 2, 5)
    ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(2)]
    outs = [torch.empty_like(x) for x in q]

    def both():
        for x, o, w in zip(q, outs, ws):
            kv.paged_attn_decode_shared(pool, 0, x, c.dtables, lens, *groups, 128 ** -0.5, o, w)
    both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for cut in (0, 15, 130, 3):
        lens.copy_(i32_dev(np.maximum(full - cut, 0)))
        both()
        torch.cuda.synchronize()
        eager = [o.clone() for o in outs]
        for o in outs:
            o.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, outs))
    assert kv.ls_device_errors() == 0


@pytest.mark.parametrize("cus", [8, 30])
def test_on_a_stream_of_few_cus(kv, cus):
    """Few workgroups: prefixes and own keys each get one at least."""
    from tests.gpu_util import cu_masked_stream, destroy_stream
    rng = np.random.default_rng(14)
    c = Cache(rng, 40 * BLOCK + rng.integers(1, 500, 7), 2, 64, [(list(range(5)), 40)])
    pool, q, out = check(kv, c, 16, "all CUs")
    made = cu_masked_stream(0, cus)
    if made is None:
        pytest.skip("no stream with a CU mask")
    stream, handle = made
    torch.cuda.synchronize()
    few = run(kv, c, pool, q, stream=stream)
    stream.synchronize()
    destroy_stream(handle)
    assert kv.ls_device_errors() == 0
    ref, mass, score, _ = decode_reference(c, 0, bits_of(q), 0.125)
    assert_within(few, ref, mass, score, 64, "%d CUs" % cus)


def test_two_calls_at_once(kv):
    """On two streams, each with a workspace of its own, over the same pool."""
    rng = np.random.default_rng(15)
    c = Cache(rng, 30 * BLOCK + rng.integers(1, 900, 24), 4, 128, [(list(range(4, 24)), 30)])
    pool = c.device(kv)
    q = [bf16_dev(W.normal_bf16(rng, (24, 32, 128))) for _ in range(2)]
    alone = [run(kv, c, pool, x) for x in q]
    n = kv.decode_shared_workspace_bytes(pool, 24, 32, 1, 20)
    ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    lens, groups, outs = i32_dev(c.lens), c.group_arrays(), [torch.empty_like(x) for x in q]
    torch.cuda.synchronize()
    for _ in range(20):
        for x, w, o, st in zip(q, ws, outs, streams):
            kv.paged_attn_decode_shared(pool, 0, x, c.dtables, lens, *groups, 128 ** -0.5, o, w, stream=st)
    torch.cuda.synchronize()
    assert kv.ls_device_errors() == 0
    assert all(torch.equal(a, b) for a, b in zip(alone, outs))


def test_half_a_thousand_sessions(kv):
    """On either side of what the smaller schedule holds."""
    rng = np.random.default_rng(16)
    for n in (511, 512, 513):
        lens = rng.integers(1, 50, n) + 3 * BLOCK
        check(kv, Cache(rng, lens, 1, 64, [(list(range(i, n, 9)), 3) for i in range(9)]), 8, "%d sessions" % n)


def bits_of(t):
    return t.view(torch.int16).cpu().numpy().view(np.uint16)
