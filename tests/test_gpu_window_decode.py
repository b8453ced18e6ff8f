"""paged_attn_decode_window against the 64-bit oracle, in pools where everything that a query does not
see is poisoned: tokens behind the window or past the end hold NaN, table entries of blocks without a
seen token name no block."""
import numpy as np
import pytest
import torch

from paper_2606_22983_amd import workloads as W
from tests.gpu_util import bf16_dev, cu_masked_stream, destroy_stream, host_bits, i32_dev
from tests.window_util import BLOCK, Sessions, assert_within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    from paper_2606_22983_amd import kv as kv_mod
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return kv_mod


class Case:
    """One windowed decode call: `lens` tokens in the pool per session, W, sinks, heads."""

    def __init__(self, kv, oracle, lens, window, sinks, hq, hkv, d, append, seed=1, extra_cols=3, layers=1, layer=0,
                 key_scale=None):
        rng = np.random.default_rng(seed)
        self.kv, self.oracle, self.window, self.sinks, self.d, self.layer = kv, oracle, window, sinks, d, layer
        self.lens = np.asarray(lens, dtype=np.int32)
        s = len(lens)
        self.pos = self.lens - (0 if append else 1)
        self.ses = Sessions(rng, self.pos, self.pos, window, sinks, hkv, d, extra_cols, layers=layers, layer=layer,
                            key_scale=key_scale)
        if append:
            for i in range(s):                        # the own token's slot is not written yet
                self.ses.poison(layer, i, [self.pos[i]], d)
        self.q = W.normal_bf16(rng, (s, hq, d))
        self.kn = W.normal_bf16(rng, (s, hkv, d)) if append else None
        self.vn = W.normal_bf16(rng, (s, hkv, d)) if append else None
        self.scale = d ** -0.5
        self.data = bf16_dev(self.ses.pool)
        nb = self.ses.pool.shape[1]
        self.pool = kv.kv_pool_create(self.data, layers, nb, hkv, d)
        self.tables, self.dlens = i32_dev(self.ses.tables), i32_dev(self.lens)
        self.dq = bf16_dev(self.q)
        self.dkn, self.dvn = (bf16_dev(self.kn), bf16_dev(self.vn)) if append else (None, None)
        size = kv.decode_window_workspace_bytes(self.pool, s, hq, self.tables.shape[1], window, sinks)
        self.ws = torch.empty(size, dtype=torch.uint8, device="cuda").random_()

    def run(self, host, stream=None, lens_host=None, workspace=None):
        out = torch.full(self.q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        self.kv.paged_attn_decode_window(self.pool, self.layer, self.dq, self.tables, self.dlens, self.window, self.sinks,
                                         self.scale, out, self.ws if workspace is None else workspace, self.dkn, self.dvn,
                                         context_lens_host=(self.lens if host else None) if lens_host is None else lens_host,
                                         stream=stream)
        torch.cuda.synchronize()
        return out

    def reference(self):
        work = self.ses.pool.copy()
        s = len(self.lens)
        if self.kn is not None:
            self.oracle.append(work, BLOCK, self.d, self.layer, self.ses.tables, np.arange(s), self.lens, self.kn, self.vn)
        ref = self.oracle.attend_window(work, BLOCK, self.d, self.layer, self.q, self.ses.tables, np.arange(s), self.pos,
                                        np.arange(s), self.scale, self.window, self.sinks)
        return work, ref

    def check(self, hosts=(False, True), what=""):
        work, (ref, mass, score) = self.reference()
        for host in hosts:
            out = self.run(host)
            assert self.kv.ls_device_errors() == 0, (what, host)
            assert_within(out, ref, mass, score, self.d, "%s %s lengths" % (what, "host" if host else "device"))
            assert np.array_equal(host_bits(self.data).reshape(work.shape), work), (what, "pool")


EDGES = [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 80, 100, 129, 300]


@pytest.mark.parametrize("append", [False, True])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 5), (2, 1), (15, 0), (16, 16), (17, 4), (64, 0), (64, 40), (100, 1),
                                          (1000, 7), (1 << 29, 0), (3, 1 << 29)])
def test_edges(kv, oracle_lib, window, sinks, append):
    lens = [x for x in EDGES] + [window % 257 + 15, window % 257 + 16, sinks % 259 + window % 257]
    lens = [max(1, x) for x in lens]
    Case(kv, oracle_lib, lens, window, sinks, 8, 2, 64, append, seed=window + sinks).check(what="W %d sinks %d" % (window, sinks))


@pytest.mark.parametrize("hq,hkv,d", [(1, 1, 64), (2, 1, 128), (4, 1, 64), (8, 1, 128), (8, 8, 64), (32, 4, 128), (16, 2, 128)])
def test_head_layouts(kv, oracle_lib, hq, hkv, d):
    Case(kv, oracle_lib, [5, 77, 130, 1040, 555], 200, 9, hq, hkv, d, True, seed=hq + d).check(what="heads %d/%d" % (hq, hkv))


# (sessions, lens from, to, window, sinks): the single-launch kernel with and without splits, the
# persistent kernel planned on the host and in the kernel, with and without the merge launch.
SHAPES = [(1, 9000, 9000, 1024, 4), (1, 5000, 5000, 4096, 16), (4, 3000, 9000, 2048, 4), (40, 100, 3000, 256, 0),
          (70, 50, 1500, 512, 4), (96, 500, 3000, 1500, 4), (300, 10, 900, 300, 20), (130, 1000, 2600, 2048, 33)]


@pytest.mark.parametrize("s,lo,hi,window,sinks", SHAPES)
@pytest.mark.parametrize("hq,hkv,d", [(16, 4, 128), (4, 4, 64)])
def test_schedules(kv, oracle_lib, s, lo, hi, window, sinks, hq, hkv, d):
    rng = np.random.default_rng(s + window)
    lens = rng.integers(lo, hi + 1, s)
    Case(kv, oracle_lib, lens, window, sinks, hq, hkv, d, bool(s % 2), seed=s).check(what="%d sessions W %d" % (s, window))


# (sessions, window): walks of one workgroup and of splits of each size, one per CU and several
SPLITS = [(1, 400), (1, 440), (1, 540), (3, 700), (6, 1300), (2, 2900), (1, 8000), (14, 1000), (20, 1500), (30, 600), (33, 2048),
          (64, 2000), (60, 900), (90, 430)]


@pytest.mark.parametrize("s,window", SPLITS)
@pytest.mark.parametrize("hq,hkv,d", [(8, 4, 128), (4, 4, 64), (2, 2, 128), (8, 2, 64)])
def test_split_sizes(kv, oracle_lib, s, window, hq, hkv, d):
    rng = np.random.default_rng(s * window)
    lens = rng.integers(window // 2, 2 * window, s)
    lens[0] = 2 * window + 7
    Case(kv, oracle_lib, lens, window, 4, hq, hkv, d, bool(window % 3), seed=s).check(what="%d sessions W %d" % (s, window))


@pytest.mark.parametrize("d", [64, 128])
def test_as_many_sessions_as_a_call_takes(kv, oracle_lib, d):
    rng = np.random.default_rng(d)
    Case(kv, oracle_lib, rng.integers(1, 500, 2048), 90, 3, 4, 1, d, True, seed=d).check(what="2048 sessions")


def test_a_table_of_two_million_tokens(kv, oracle_lib):
    """Positions and table columns far past the blocks that a call may read (16384)."""
    cols = 1 << 17
    Case(kv, oracle_lib, [cols * BLOCK - 1, 5, 100000], 700, 20, 8, 2, 128, True, seed=41, extra_cols=0).check(what="long cache")


@pytest.mark.parametrize("host", [False, True])
def test_small_workspace_runs_the_persistent_kernel(kv, oracle_lib, host):
    """The least workspace a call takes leaves the single-launch schedule no room."""
    c = Case(kv, oracle_lib, [3000, 4000, 800, 2222], 1200, 4, 16, 4, 128, True, seed=3)
    _, (ref, mass, score) = c.reference()
    for size in (c.ws.numel(), c.ws.numel() // 2, c.ws.numel() // 4, 1 << 14):
        try:
            out = c.run(host, workspace=c.ws[:size])
        except kv.LiveServeError as e:
            assert e.status == kv.LS_ENOMEM
            break
        assert kv.ls_device_errors() == 0
        assert_within(out, ref, mass, score, 128, "workspace of %d" % size)


@pytest.mark.parametrize("shape", ["rising", "falling", "spike"])
def test_peaky_scores(kv, oracle_lib, shape):
    def scale(t, n):
        x = t / max(n - 1, 1)
        return {"rising": 1 + 9 * x, "falling": 10 - 9 * x, "spike": np.where(t == n - 5, 16.0, 1.0)}[shape]
    Case(kv, oracle_lib, [40, 700, 1500, 3000], 1024, 4, 8, 1, 128, False, seed=11, key_scale=scale).check(what=shape)


def test_window_that_covers_everything_is_plain_decode(kv, oracle_lib):
    c = Case(kv, oracle_lib, [1, 100, 777, 2000], 2001, 0, 16, 4, 128, True, seed=5)
    ws = torch.empty(kv.decode_workspace_bytes(c.pool, 4, 16, c.tables.shape[1]), dtype=torch.uint8, device="cuda")
    for host in (None, c.lens):
        plain = torch.empty_like(c.dq)
        kv.paged_attn_decode(c.pool, 0, c.dq, c.tables, c.dlens, c.scale, plain, ws, c.dkn, c.dvn, context_lens_host=host)
        got = torch.empty_like(c.dq)
        kv.paged_attn_decode_window(c.pool, 0, c.dq, c.tables, c.dlens, 2001, 0, c.scale, got,
                                    torch.empty_like(ws).resize_(ws.numel() * 2), c.dkn, c.dvn, context_lens_host=host)
        torch.cuda.synchronize()
        assert (plain.float() - got.float()).abs().max() < 2.0 ** -5
    assert kv.ls_device_errors() == 0


def test_layer_offset_and_other_layers_stay(kv, oracle_lib):
    c = Case(kv, oracle_lib, [50, 333], 64, 3, 8, 2, 64, True, seed=6, layers=3, layer=1)
    c.check(what="layer 1 of 3")


def test_runs_repeat_bit_for_bit(kv, oracle_lib):
    for host in (False, True):
        c = Case(kv, oracle_lib, np.random.default_rng(9).integers(1, 5000, 33), 1024, 4, 32, 4, 128, False, seed=9)
        a = c.run(host)
        for _ in range(3):
            assert torch.equal(a.view(torch.int16), c.run(host).view(torch.int16))


def test_other_stream_and_cu_masked_stream(kv, oracle_lib):
    c = Case(kv, oracle_lib, [900, 4000, 2500, 20, 1300], 1000, 4, 32, 4, 128, True, seed=8)
    _, (ref, mass, score) = c.reference()
    assert_within(c.run(True, stream=torch.cuda.Stream()), ref, mass, score, 128, "side stream")
    made = cu_masked_stream(0, 32)
    if made is not None:
        st, handle = made
        for host in (False, True):
            assert_within(c.run(host, stream=st), ref, mass, score, 128, "32 CUs")
        torch.cuda.synchronize()
        destroy_stream(handle)
    assert kv.ls_device_errors() == 0


def test_bad_lengths_and_ids_are_flagged(kv, oracle_lib):
    c = Case(kv, oracle_lib, [100, 200, 300], 64, 4, 8, 2, 64, False, seed=12)
    cap = c.tables.shape[1] * BLOCK
    c.dlens.copy_(i32_dev([0, 200, -5]))
    out = c.run(False)
    assert kv.ls_device_errors() == kv.LS_DEVERR_LENGTH
    assert (out[0] == 0).all() and (out[2] == 0).all() and torch.isfinite(out[1].float()).all()
    # a length past the table is clipped to it: its window's blocks are stale ids here
    c.dlens.copy_(i32_dev([100, cap + 1, 2**31 - 1]))
    c.run(False)
    assert kv.ls_device_errors() & kv.LS_DEVERR_LENGTH
    c.dlens.copy_(i32_dev(c.lens))
    keep = c.tables.clone()
    c.tables[1, 199 // BLOCK] = c.pool.num_blocks
    for host in (False, True):
        c.run(host)
        assert kv.ls_device_errors() == kv.LS_DEVERR_BLOCK_ID
    c.tables.copy_(keep)
    c.check(what="afterwards")


def test_host_lengths_that_differ_are_flagged(kv, oracle_lib):
    """Device lengths of more keys than the host's plan covers (its block columns may hold stale ids)."""
    c = Case(kv, oracle_lib, [600, 600], 512, 0, 8, 2, 128, False, seed=13)
    c.run(True, lens_host=np.array([600, 20], dtype=np.int32))
    bits = kv.ls_device_errors()
    assert bits & kv.LS_DEVERR_LENGTH and not bits & ~(kv.LS_DEVERR_LENGTH | kv.LS_DEVERR_BLOCK_ID)


def test_captured_steps_replay(kv, oracle_lib):
    c = Case(kv, oracle_lib, np.random.default_rng(2).integers(50, 3000, 24), 700, 4, 16, 2, 128, True, seed=14)
    out = torch.empty_like(c.dq)

    def step():
        kv.paged_attn_decode_window(c.pool, 0, c.dq, c.tables, c.dlens, c.window, c.sinks, c.scale, out, c.ws, c.dkn, c.dvn)
    step()
    torch.cuda.synchronize()
    eager = out.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(3):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), eager.view(torch.int16))
    assert kv.ls_device_errors() == 0
