"""kv_tables_update and kv_append against the oracle: equal to the last value."""
import numpy as np
import pytest
import torch

from paper_2606_22983_amd import workloads as W
from tests.gpu_util import bf16_dev, host_bits, i32_dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    from paper_2606_22983_amd import kv as kv_mod
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return kv_mod


def i64_dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int64)).cuda()


class Step:
    """A step's inputs: sessions of `lens` tokens, `new` more; a ring with `slack` more ids than the step takes."""

    def __init__(self, kv, lens, new, window=0, sinks=0, ring=True, pad=0, slack=0, start=0, extra_cols=2, seed=1):
        rng = np.random.default_rng(seed)
        self.kv, self.window, self.sinks = kv, window, sinks
        self.lens, self.new = np.asarray(lens, dtype=np.int32), np.asarray(new, dtype=np.int32)
        s = len(self.lens)
        total = self.lens.astype(np.int64) + self.new
        have, want = -(-self.lens.astype(np.int64) // 16), -(-total // 16)
        cols = max(1, int(want.max(initial=0))) + extra_cols
        held, need = int(have.sum()), int((want - have).sum())
        self.nb = held + need + slack + 3
        perm = rng.permutation(self.nb).astype(np.int32)
        self.tables = np.full((s, cols), -9, dtype=np.int32)
        at = 0
        for i in range(s):
            n = int(have[i] if ring else want[i])
            self.tables[i, :n] = perm[at:at + n]
            at += n
        self.ring = self.counts = None
        if ring:
            size = 2 * self.nb
            self.ring = np.full(size, -5, dtype=np.int32)
            free = perm[held:held + need + slack]
            self.ring[(start + np.arange(len(free))) % size] = free
            self.counts = np.array([start, start + len(free)], dtype=np.int64)
        self.total = int(self.new.sum()) + pad
        self.max_new = int(self.new.max(initial=0))
        self.pool = kv.kv_pool_create(self._mem(), 1, self.nb, 1, 64)

    def _mem(self):
        return torch.empty(self.kv.ls_kv_pool_bytes(1, self.nb, 1, 64), dtype=torch.uint8, device="cuda")

    def upload(self):
        dev = {"lens": i32_dev(self.lens), "new": i32_dev(self.new), "tables": i32_dev(self.tables),
               "next": torch.full((len(self.lens),), -77, dtype=torch.int32, device="cuda"),
               "cu": torch.full((len(self.lens) + 1,), -77, dtype=torch.int32, device="cuda"),
               "reused": torch.full((len(self.lens),), -77, dtype=torch.int32, device="cuda"),
               "slots": torch.full((self.total,), -77, dtype=torch.int64, device="cuda"),
               "ring": None, "counts": None, "next_counts": None}
        if self.ring is not None:
            dev.update(ring=i32_dev(self.ring), counts=i64_dev(self.counts), next_counts=i64_dev([-77, -77]))
        return dev

    def call(self, t, in_place=False, max_new=None):
        self.kv.kv_tables_update(self.pool, t["lens"], t["new"], self.max_new if max_new is None else max_new, t["tables"],
                                 t["lens"] if in_place else t["next"], t["cu"], t["reused"], t["slots"],
                                 free_ring=t["ring"], free_counts=t["counts"],
                                 next_counts=t["counts"] if in_place else t["next_counts"], window=self.window,
                                 sinks=self.sinks)

    def check(self, oracle, what=""):
        want = oracle.tables_step(self.lens, self.new, self.tables, self.ring, self.counts, self.window, self.sinks, self.total)
        for repeat in (False, True):
            t = self.upload()
            self.call(t)
            if repeat:                                  # inputs and outputs are apart: again, the same
                self.call(t)
            torch.cuda.synchronize()
            assert self.kv.ls_device_errors() == 0, what
            self.same(t, want, what)
            assert np.array_equal(t["lens"].cpu().numpy(), self.lens) and np.array_equal(t["next"].cpu().numpy(), want["next"])
            if self.ring is not None:
                assert np.array_equal(t["counts"].cpu().numpy(), self.counts)
                assert np.array_equal(t["next_counts"].cpu().numpy(), want["counts"]), what
        t = self.upload()
        self.call(t, in_place=True)
        torch.cuda.synchronize()
        self.same(t, want, what + " in place")
        assert np.array_equal(t["lens"].cpu().numpy(), want["next"])
        if self.ring is not None:
            assert np.array_equal(t["counts"].cpu().numpy(), want["counts"])
        return want

    def same(self, t, want, what):
        assert np.array_equal(t["tables"].cpu().numpy(), want["tables"]), what
        assert np.array_equal(t["slots"].cpu().numpy(), want["slots"]), what
        assert np.array_equal(t["cu"].cpu().numpy(), want["cu"]), what
        assert np.array_equal(t["reused"].cpu().numpy(), self.lens), what
        if self.ring is not None:
            assert np.array_equal(t["ring"].cpu().numpy(), want["ring"]), what


CASES = [
    ([0], [0]), ([0], [1]), ([15], [1]), ([16], [1]), ([17], [1]), ([0], [16]), ([0], [17]), ([3], [1000]),
    (list(range(64)), [1] * 64), (list(range(0, 300)), [i % 2 for i in range(300)]), ([5, 0, 31, 16], [0, 40, 1, 300]),
]


@pytest.mark.parametrize("lens,new", CASES)
@pytest.mark.parametrize("window,sinks,ring", [(0, 0, False), (0, 0, True), (1, 0, True), (16, 0, True), (17, 1, True), (40, 33, True),
                                               (100, 16, True), (1 << 29, 1 << 29, True)])
def test_steps(kv, oracle_lib, lens, new, window, sinks, ring):
    Step(kv, lens, new, window, sinks, ring, pad=3, slack=2, start=7).check(oracle_lib, "W %d sinks %d" % (window, sinks))


# small and large steps: a decode step, more sessions than a workgroup has threads, turns of many rows
LARGE = [(256, 1, 1, 0, 5000, 1024), (1500, 1, 1, 0, 300, 64), (3000, 0, 3, 0, 100, 16), (32, 256, 2048, 2000, 9000, 1024), (1, 20000, 20000, 5, 5, 0),
         (1, 9000, 9000, 0, 0, 256), (200, 1, 90, 0, 700, 128), (2, 1, 5000, 100, 200, 0),
         (256, 2, 2, 0, 90, 32), (256, 3, 9, 0, 90, 32), (257, 0, 2, 0, 90, 32), (1024, 1, 1, 0, 90, 32), (1025, 0, 9, 0, 90, 32),
         (4096, 1, 1, 0, 40, 16), (4097, 0, 1, 0, 40, 16), (9000, 0, 3, 0, 40, 16)]


@pytest.mark.parametrize("s,lo,hi,clo,chi,window", LARGE)
def test_large_steps(kv, oracle_lib, s, lo, hi, clo, chi, window):
    rng = np.random.default_rng(s + hi)
    Step(kv, rng.integers(clo, chi + 1, s), rng.integers(lo, hi + 1, s), window, 4, True, pad=50, slack=9, start=(1 << 40) + 3,
         seed=s).check(oracle_lib, "%d sessions" % s)


def test_ring_that_wraps_and_a_ring_without_slack(kv, oracle_lib):
    for start in (0, 1, 50, 10**12 + 17):
        Step(kv, [100, 200, 300], [40, 1, 77], 64, 2, True, slack=0, start=start).check(oracle_lib, "start %d" % start)


def test_table_columns_over_a_long_cache(kv, oracle_lib):
    """A session near the end of a table of 2^20 blocks."""
    Step(kv, [(1 << 20) * 16 - 40, 3], [40, 20], 4096, 4, True, extra_cols=0).check(oracle_lib, "long cache")


REFUSED = [
    ("a negative length", dict(lens=[5, -1, 7]), "LENGTH"),
    ("a negative turn", dict(new=[1, -1, 1]), "LENGTH"),
    ("a turn over max_new_len", dict(new=[1, 9, 1], max_new=8), "LENGTH"),
    ("a table that is too short", dict(lens=[5, 10**6, 7]), "LENGTH"),
    ("more rows than slots", dict(new=[3, 3, 3], total=8), "LENGTH"),
    ("too few free blocks", dict(new=[3, 60, 3], counts=[4, 6]), "FREE"),
    ("counters that cannot be", dict(counts=[9, 4]), "FREE"),
    ("a ring fuller than it is", dict(counts=[0, 10**9]), "FREE"),
    ("negative counters", dict(counts=[-5, 100]), "FREE"),
    ("no room to give blocks back", dict(lens=[30, 0, 300], new=[1, 1, 160], counts=[0, 71], ring=range(72), total=200, max_new=200), "FREE"),
]


@pytest.mark.parametrize("what,change,bit", REFUSED, ids=[r[0] for r in REFUSED])
def test_steps_are_refused_as_a_whole(kv, oracle_lib, what, change, bit):
    p = Step(kv, [5, 40, 7], [1, 1, 12], 16, 0, True, pad=100, slack=20, start=3, extra_cols=30)
    for k, v in change.items():
        if k == "total":
            p.total = v
        elif k == "max_new":
            p.max_new = v
        else:
            setattr(p, k, np.asarray(v, dtype=np.int64 if k == "counts" else np.int32))
    t = p.upload()
    p.call(t, max_new=change.get("max_new", 100))
    torch.cuda.synchronize()
    assert kv.ls_device_errors() == (kv.LS_DEVERR_LENGTH if bit == "LENGTH" else kv.LS_DEVERR_FREE_LIST)
    assert (t["cu"] == 0).all() and (t["slots"] == -1).all()
    for k, want in (("tables", p.tables), ("ring", p.ring), ("next", p.lens), ("next_counts", p.counts), ("reused", p.lens)):
        assert np.array_equal(t[k].cpu().numpy(), want), k


def test_ids_outside_the_pool_are_flagged(kv, oracle_lib):
    p = Step(kv, [5, 16], [4, 20], 0, 0, True, slack=4)
    p.tables[0, 0] = p.nb                              # the open block of session 0
    p.ring[1] = -4                                     # the second block that session 1 opens
    t = p.upload()
    p.call(t)
    torch.cuda.synchronize()
    assert kv.ls_device_errors() == kv.LS_DEVERR_BLOCK_ID
    slots = t["slots"].cpu().numpy()
    assert (slots[:4] == -1).all() and (slots[4:20] >= 0).all() and (slots[20:24] == -1).all()


def test_captured_steps_advance(kv, oracle_lib):
    """A captured step that advances lengths and counters in place, replayed: each replay is the oracle's next step."""
    p = Step(kv, [0, 30, 47, 200], [1, 1, 1, 1], 40, 4, True, pad=1, slack=30, extra_cols=6)
    t = p.upload()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        p.call(t, in_place=True)
    tables, ring, counts, lens = p.tables, p.ring, p.counts, p.lens
    for _ in range(60):
        g.replay()
        want = oracle_lib.tables_step(lens, p.new, tables, ring, counts, 40, 4, p.total)
        torch.cuda.synchronize()
        for k in ("tables", "slots", "ring", "counts"):
            assert np.array_equal(t[k].cpu().numpy(), want[k]), k
        assert np.array_equal(t["lens"].cpu().numpy(), want["next"]) and np.array_equal(t["reused"].cpu().numpy(), lens)
        tables, ring, counts, lens = want["tables"], want["ring"], want["counts"], want["next"]
    assert kv.ls_device_errors() == 0


# ---- kv_append


def append_case(kv, oracle, slots, hkv, d, fused, nb, layers=1, layer=0, seed=1, host=False):
    rng = np.random.default_rng(seed)
    slots = np.asarray(slots, dtype=np.int64)
    t = len(slots)
    pool = rng.integers(0, 1 << 16, (layers, nb, 2, hkv, 16 * d), dtype=np.uint16)
    data = bf16_dev(pool)
    handle = kv.kv_pool_create(data, layers, nb, hkv, d)
    kn, vn = (rng.integers(0, 1 << 16, (t, hkv, d), dtype=np.uint16) for _ in range(2))      # bits, NaN among them
    if fused:
        wide = torch.zeros((t, 3 * hkv + 1, d), dtype=torch.int16, device="cuda")
        wide[:, hkv:2 * hkv] = bf16_dev(kn).view(torch.int16)
        wide[:, 2 * hkv + 1:] = bf16_dev(vn).view(torch.int16)
        dk, dv = wide[:, hkv:2 * hkv], wide[:, 2 * hkv + 1:]
    else:
        dk, dv = bf16_dev(kn), bf16_dev(vn)
    kv.kv_append(handle, layer, dk, dv, i64_dev(slots), slot_map_host=slots if host else None)
    torch.cuda.synchronize()
    assert kv.ls_device_errors() == 0
    want = pool.copy()
    oracle.append_slots(want, 16, d, layer, kn, vn, slots)
    assert np.array_equal(host_bits(data).reshape(want.shape), want)


def runs(rng, nb, lens, shift=True):
    """Slot runs of sessions: consecutive tokens over shuffled blocks, each run starting anywhere in its first block."""
    out, ids = [], rng.permutation(nb)
    for n in lens:
        off = int(rng.integers(0, 16)) if shift else 0
        k = (off + n + 15) // 16
        mine, ids = ids[:k], ids[k:]
        p = off + np.arange(n)
        out.append(mine[p // 16] * 16 + p % 16)
    return np.concatenate(out) if out else np.empty(0, dtype=np.int64)


@pytest.mark.parametrize("hkv,d", [(1, 64), (2, 128), (3, 64), (8, 128), (4, 128), (5, 128)])
@pytest.mark.parametrize("fused", [False, True])
def test_append_runs(kv, oracle_lib, hkv, d, fused):
    rng = np.random.default_rng(hkv)
    for lens in ([1], [16], [15, 1, 16, 17], [64] * 5, [1] * 40, [333], [7, 8, 9, 200, 31]):
        append_case(kv, oracle_lib, runs(rng, 90, lens), hkv, d, fused, 90, host=True)
        append_case(kv, oracle_lib, runs(rng, 90, lens, shift=False), hkv, d, fused, 90)


@pytest.mark.parametrize("d", [64, 128])
def test_append_in_any_order_and_with_rows_left_out(kv, oracle_lib, d):
    rng = np.random.default_rng(d)
    every = rng.permutation(40 * 16)
    append_case(kv, oracle_lib, every[:100], 2, d, False, 40)
    append_case(kv, oracle_lib, every, 3, d, True, 40)
    append_case(kv, oracle_lib, np.arange(500)[::-1], 2, d, False, 40)                       # descending
    append_case(kv, oracle_lib, np.arange(0, 640, 2), 2, d, False, 40)                       # every other slot
    some = runs(rng, 40, [100, 50, 200])
    some[rng.random(len(some)) < 0.3] = -1
    some[60:90] = -(1 << 40)
    append_case(kv, oracle_lib, some, 2, d, True, 40, layers=3, layer=2)
    append_case(kv, oracle_lib, np.full(33, -1), 2, d, False, 40)
    swapped = np.arange(320).reshape(-1, 2)[:, ::-1].reshape(-1)                             # pairs the wrong way round
    append_case(kv, oracle_lib, swapped, 1, d, False, 40)


@pytest.mark.parametrize("hkv,d", [(32, 64), (32, 128), (7, 64), (7, 128)])
@pytest.mark.parametrize("rows", [40, 900, 4000, 15000])
def test_append_row_counts(kv, oracle_lib, hkv, d, rows):
    """From few rows, a few per workgroup, to many: runs of turns, lone slots and rows left out, mixed."""
    if rows * hkv > 130000:
        rows = 4001
    rng = np.random.default_rng(rows + hkv)
    lens, left = [], rows
    while left > 0:
        lens.append(min(left, int(rng.choice([1, 2, 15, 16, 17, 40, 200]))))
        left -= lens[-1]
    nb = sum((n + 30) // 16 for n in lens)
    slots = runs(rng, nb, lens)
    slots[rng.random(rows) < 0.02] = -1
    append_case(kv, oracle_lib, slots, hkv, d, rows % 2 == 0, nb, host=True)


def test_append_large_and_slots_past_the_pool(kv, oracle_lib):
    rng = np.random.default_rng(3)
    append_case(kv, oracle_lib, runs(rng, 900, rng.integers(1, 700, 20)), 4, 128, True, 900)
    nb = 4
    data = torch.zeros((1, nb, 2, 2, 16 * 64), dtype=torch.bfloat16, device="cuda")
    pool = kv.kv_pool_create(data, 1, nb, 2, 64)
    rows = torch.ones((20, 2, 64), dtype=torch.bfloat16, device="cuda")
    slots = torch.arange(50, 70, device="cuda")
    kv.kv_append(pool, 0, rows, rows, slots)
    torch.cuda.synchronize()
    assert kv.ls_device_errors() == kv.LS_DEVERR_BLOCK_ID
    assert int((data != 0).sum()) == 14 * 2 * 2 * 64                                         # slots 50 .. 63
    slots[3] = (1 << 62) + 5
    kv.kv_append(pool, 0, rows, rows, slots)
    assert kv.ls_device_errors() == kv.LS_DEVERR_BLOCK_ID
    with pytest.raises(kv.LiveServeError):
        kv.kv_append(pool, 0, rows, rows, slots, slot_map_host=slots.cpu())


def test_append_two_streams_into_one_block(kv, oracle_lib):
    """Different slots of the same blocks, written from two streams at once."""
    data = torch.zeros((1, 64, 2, 2, 16 * 128), dtype=torch.bfloat16, device="cuda")
    pool = kv.kv_pool_create(data, 1, 64, 2, 128)
    rng = np.random.default_rng(4)
    slots = rng.permutation(64 * 16)
    rows = [W.normal_bf16(rng, (1024, 2, 128)) for _ in range(2)]
    dk, dv = (bf16_dev(r) for r in rows)
    a, b = i64_dev(np.where(slots % 2 == 0, slots, -1)), i64_dev(np.where(slots % 2 == 1, slots, -1))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for st, m in zip(streams, (a, b)):
        kv.kv_append(pool, 0, dk, dv, m, stream=st)
    torch.cuda.synchronize()
    assert kv.ls_device_errors() == 0
    want = np.zeros((1, 64, 2, 2, 16 * 128), dtype=np.uint16)
    oracle_lib.append_slots(want, 16, 128, 0, rows[0], rows[1], slots)
    assert np.array_equal(host_bits(data).reshape(want.shape), want)
