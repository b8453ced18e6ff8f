"""paged_attn_prefill_window against the 64-bit oracle, in pools where every token that no row of the
turn sees holds NaN and table entries of blocks without a seen token name no block."""
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
    """One windowed prefill call: (n, c) per session."""

    def __init__(self, kv, oracle, turns, window, sinks, hq, hkv, d, append, seed=1, extra_cols=2, layers=1, layer=0,
                 key_scale=None):
        rng = np.random.default_rng(seed)
        self.kv, self.oracle, self.window, self.sinks, self.d, self.layer = kv, oracle, window, sinks, d, layer
        self.n, self.c = (np.array(x, dtype=np.int32) for x in zip(*turns))
        self.cu = np.concatenate([[0], np.cumsum(self.n)]).astype(np.int32)
        self.ses = Sessions(rng, self.c, self.c + self.n - 1, window, sinks, hkv, d, extra_cols, layers=layers, layer=layer,
                            key_scale=key_scale)
        total = int(self.cu[-1])
        self.who = np.repeat(np.arange(len(self.n)), self.n)
        self.pos = (self.c[self.who] + np.arange(total) - self.cu[self.who]).astype(np.int32)
        self.kn = self.vn = None
        if append:
            for i in range(len(self.n)):
                if self.n[i]:
                    self.ses.poison(layer, i, np.arange(self.c[i], self.c[i] + self.n[i]), d)
            self.kn, self.vn = W.normal_bf16(rng, (total, hkv, d)), W.normal_bf16(rng, (total, hkv, d))
        self.q = W.normal_bf16(rng, (total, hq, d))
        self.scale = d ** -0.5
        self.data = bf16_dev(self.ses.pool)
        self.pool = kv.kv_pool_create(self.data, layers, self.ses.pool.shape[1], hkv, d)
        self.tables, self.dcu, self.dctx = i32_dev(self.ses.tables), i32_dev(self.cu), i32_dev(self.c)
        self.dq = bf16_dev(self.q)
        self.dkn, self.dvn = (bf16_dev(self.kn), bf16_dev(self.vn)) if append else (None, None)
        self.lens_host = np.ascontiguousarray(np.stack([self.n, self.c], 1), dtype=np.int32)
        self.ws = torch.empty(kv.PREFILL_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")

    def run(self, mode, stream=None):
        out = torch.full(self.q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
        ws = {"device": None, "host": None, "counters": self.ws[:256], "full": self.ws}[mode]
        if ws is not None:
            ws.random_()
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        self.kv.paged_attn_prefill_window(self.pool, self.layer, self.dq, self.dcu, self.dctx, int(self.n.max()), self.tables,
                                          self.window, self.sinks, self.scale, out, self.dkn, self.dvn,
                                          lens_host=None if mode == "device" else self.lens_host, workspace=ws,
                                          stream=stream)
        torch.cuda.synchronize()
        return out

    def reference(self, rows=None):
        work = self.ses.pool.copy()
        if self.kn is not None:
            self.oracle.append(work, BLOCK, self.d, self.layer, self.ses.tables, self.who, self.pos, self.kn, self.vn)
        rows = np.arange(len(self.pos)) if rows is None else rows
        ref = self.oracle.attend_window(work, BLOCK, self.d, self.layer, self.q, self.ses.tables, self.who[rows],
                                        self.pos[rows], rows, self.scale, self.window, self.sinks)
        return work, ref

    def check(self, modes=("device", "host", "counters", "full"), what="", rows=None):
        work, (ref, mass, score) = self.reference(rows)
        for mode in modes:
            out = self.run(mode)
            assert self.kv.ls_device_errors() == 0, (what, mode)
            assert torch.isfinite(out.float()).all(), (what, mode)
            out = out if rows is None else out[torch.from_numpy(rows).cuda()]
            assert_within(out, ref, mass, score, self.d, "%s %s" % (what, mode))
            assert np.array_equal(host_bits(self.data).reshape(work.shape), work), (what, mode, "pool")


WINDOWS = [(1, 0), (1, 3), (2, 0), (15, 1), (16, 0), (17, 16), (31, 33), (64, 0), (65, 70), (100, 4), (300, 0),
           (1 << 29, 0), (5, 1 << 29)]


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("hq,hkv,d,append", [(8, 1, 64, True), (2, 2, 64, False), (4, 2, 128, True), (8, 2, 128, False)])
def test_edges(kv, oracle_lib, window, sinks, hq, hkv, d, append):
    turns = [(1, 0), (40, 0), (33, 15), (1, 16), (17, 17), (100, 63), (2, 300), (130, 257), (31, 1), (64, 128), (0, 40)]
    Case(kv, oracle_lib, turns, window, sinks, hq, hkv, d, append, seed=window + sinks + d).check(
        what="W %d sinks %d" % (window, sinks))


@pytest.mark.parametrize("hq,hkv,d", [(1, 1, 128), (2, 1, 64), (16, 4, 64), (32, 4, 128), (8, 8, 64), (8, 8, 128)])
def test_head_layouts(kv, oracle_lib, hq, hkv, d):
    Case(kv, oracle_lib, [(70, 500), (3, 1000), (301, 20)], 200, 9, hq, hkv, d, True, seed=hq + d).check(
        what="heads %d/%d" % (hq, hkv))


@pytest.mark.parametrize("turns,window,sinks,hq,hkv,d", [
    ([(301, 9043)], 2048, 4, 32, 4, 128),                                 # split over the keys
    ([(600, 3000), (20, 5000), (900, 100)], 1500, 20, 8, 1, 128),
    ([(500, 700), (700, 0)], 256, 0, 4, 4, 64),
    ([(50, 4000)] * 12, 1024, 4, 8, 2, 128),
    ([(9, 2000)] * 20, 700, 1, 8, 8, 64),                                 # turns of half a query tile and less
])
def test_schedules(kv, oracle_lib, turns, window, sinks, hq, hkv, d):
    c = Case(kv, oracle_lib, turns, window, sinks, hq, hkv, d, True, seed=len(turns))
    rows = np.unique(np.concatenate([c.cu[:-1], c.cu[1:] - 1, np.random.default_rng(1).integers(0, c.cu[-1], 120)]))
    c.check(what="%d turns W %d" % (len(turns), window), rows=rows)


@pytest.mark.parametrize("sessions,hkv", [(70, 8), (40, 8), (300, 1)])
def test_many_pairs(kv, oracle_lib, sessions, hkv):
    """More (session, KV head) pairs than a host plan holds (256), or than the kernel schedules (512)."""
    rng = np.random.default_rng(sessions)
    turns = [(int(rng.integers(1, 40)), int(rng.integers(0, 300))) for _ in range(sessions)]
    c = Case(kv, oracle_lib, turns, 100, 5, 2 * hkv, hkv, 64, True, seed=sessions)
    c.check(what="%d sessions of %d heads" % (sessions, hkv))


def test_a_table_of_two_million_tokens(kv, oracle_lib):
    cols = 1 << 17
    c = Case(kv, oracle_lib, [(50, cols * BLOCK - 50), (20, 300)], 300, 4, 8, 2, 64, True, seed=41, extra_cols=0)
    assert c.tables.shape[1] == cols
    c.check(what="long cache")


@pytest.mark.parametrize("shape", ["rising", "falling", "spike", "sinks", "own"])
def test_peaky_scores(kv, oracle_lib, shape):
    """Keys far larger than the row's own (whose score the running maximum starts from), or far smaller."""
    def scale(t, n):
        x = t / max(n - 1, 1)
        return {"rising": 1 + 9 * x, "falling": 10 - 9 * x, "spike": np.where(t % 97 == 5, 16.0, 1.0),
                "sinks": np.where(t < 4, 20.0, 0.5), "own": np.where(t >= n - 40, 12.0, 0.2)}[shape]
    c = Case(kv, oracle_lib, [(90, 1300), (40, 100), (300, 3)], 512, 4, 8, 1, 128, False, seed=11, key_scale=scale)
    c.check(what=shape)


@pytest.mark.parametrize("mode", ["device", "host", "full"])
def test_infinite_keys(kv, oracle_lib, mode):
    """A row whose own key scores -inf (an infinite K) starts from its first finite score, in every part of the keys."""
    c = Case(kv, oracle_lib, [(20, 2500)], 2048, 4, 8, 1, 128, False, seed=21)
    d = 128
    # own key of row 7: K = -inf in one dimension where q is 1, K's other dimensions 0
    p = 2500 + 7
    b, o = c.ses.tables[0, p // BLOCK], p % BLOCK
    kt = c.ses.pool[0, :, 0].reshape(-1, 1, d // 8, BLOCK, 8)
    kt[b, 0, :, o] = 0
    kt[b, 0, 0, o, 0] = 0xFF80                                      # -inf
    c.q[7:, :, 0] = 0x3F80                                          # 1.0: rows that see the key score -inf with it
    c.q[:7, :, 0] = 0x3F80
    c.data.copy_(bf16_dev(c.ses.pool))
    c.dq.copy_(bf16_dev(c.q))
    out = c.run(mode)
    finite = c.ses.pool.copy()
    finite[0, :, 0].reshape(-1, 1, d // 8, BLOCK, 8)[b, 0, 0, o, 0] = 0xD000      # about -8.6e9: weight 0 all the same
    ref, mass, score = c.oracle.attend_window(finite, BLOCK, d, 0, c.q, c.ses.tables, c.who, c.pos, np.arange(20), c.scale,
                                              2048, 4)
    g = out.float().cpu().numpy()
    assert np.isfinite(g).all()
    # (score is that key's: its size plays no part in the others' error)
    score = np.full_like(score, 60.0)
    assert_within(out, ref, mass, score, d, "own key at -inf, " + mode)


def test_chunks_give_the_whole_turn(kv, oracle_lib):
    """A turn in two chunks, the second over the first's tokens, is the turn in one."""
    c = Case(kv, oracle_lib, [(200, 333)], 150, 4, 8, 2, 64, True, seed=31)
    whole = c.run("device")
    out = torch.empty_like(whole)
    for lo, hi in ((0, 77), (77, 200)):
        kv.paged_attn_prefill_window(c.pool, 0, c.dq[lo:hi], i32_dev([0, hi - lo]), i32_dev([333 + lo]), hi - lo, c.tables, 150, 4,
                                     c.scale, out[lo:hi], c.dkn[lo:hi], c.dvn[lo:hi])
    torch.cuda.synchronize()
    assert kv.ls_device_errors() == 0
    _, (ref, mass, score) = c.reference()
    assert_within(out, ref, mass, score, 64, "two chunks")
    assert_within(whole, ref, mass, score, 64, "one")


def test_one_token_is_the_decode_step(kv, oracle_lib):
    c = Case(kv, oracle_lib, [(1, 700), (1, 5), (1, 0), (1, 2000)], 512, 4, 16, 2, 128, True, seed=32)
    out = c.run("device")
    dec = torch.empty_like(out)
    ws = torch.empty(kv.decode_window_workspace_bytes(c.pool, 4, 16, c.tables.shape[1], 512, 4), dtype=torch.uint8, device="cuda")
    kv.paged_attn_decode_window(c.pool, 0, c.dq, c.tables, c.dctx, 512, 4, c.scale, dec, ws, c.dkn, c.dvn)
    torch.cuda.synchronize()
    _, (ref, mass, score) = c.reference()
    assert_within(out, ref, mass, score, 128, "prefill of one token")
    assert_within(dec, ref, mass, score, 128, "decode")


def test_rows_behind_the_last_session_stay(kv, oracle_lib):
    c = Case(kv, oracle_lib, [(37, 100), (5, 60)], 64, 2, 8, 2, 64, False, seed=33)
    q = torch.cat([c.dq, torch.full((11,) + c.dq.shape[1:], float("nan"), dtype=torch.bfloat16, device="cuda")])
    out = torch.full_like(q, 7.0)
    kv.paged_attn_prefill_window(c.pool, 0, q, c.dcu, c.dctx, 37, c.tables, 64, 2, c.scale, out)
    torch.cuda.synchronize()
    assert kv.ls_device_errors() == 0
    _, (ref, mass, score) = c.reference()
    assert_within(out[:42], ref, mass, score, 64, "padded batch")
    assert (out[42:] == 7.0).all()


def test_other_stream_and_cu_masked_stream(kv, oracle_lib):
    c = Case(kv, oracle_lib, [(301, 3000), (50, 900)], 700, 4, 16, 2, 128, True, seed=34)
    _, (ref, mass, score) = c.reference()
    assert_within(c.run("full", stream=torch.cuda.Stream()), ref, mass, score, 128, "side stream")
    made = cu_masked_stream(0, 32)
    if made is not None:
        st, handle = made
        for mode in ("device", "full"):
            assert_within(c.run(mode, stream=st), ref, mass, score, 128, "32 CUs")
        torch.cuda.synchronize()
        destroy_stream(handle)
    assert kv.ls_device_errors() == 0


def test_runs_repeat_bit_for_bit_and_captured(kv, oracle_lib):
    c = Case(kv, oracle_lib, [(301, 3000), (50, 900), (7, 20)], 700, 4, 16, 2, 128, True, seed=35)
    for mode in ("device", "full"):
        a = c.run(mode)
        assert torch.equal(a.view(torch.int16), c.run(mode).view(torch.int16))
        out = torch.empty_like(a)
        ws = c.ws if mode == "full" else None

        def call():
            kv.paged_attn_prefill_window(c.pool, 0, c.dq, c.dcu, c.dctx, 301, c.tables, 700, 4, c.scale, out, c.dkn, c.dvn,
                                         lens_host=c.lens_host if ws is not None else None, workspace=ws)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        for _ in range(3):
            out.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out.view(torch.int16), a.view(torch.int16)), mode
    assert kv.ls_device_errors() == 0


def test_bad_lengths_and_ids_are_flagged(kv, oracle_lib):
    c = Case(kv, oracle_lib, [(20, 100), (30, 50)], 64, 4, 8, 2, 64, False, seed=36)
    c.dctx.copy_(i32_dev([-3, 50]))
    c.run("device")
    assert kv.ls_device_errors() & kv.LS_DEVERR_LENGTH
    c.dctx.copy_(i32_dev([c.tables.shape[1] * BLOCK, 50]))
    c.run("device")
    assert kv.ls_device_errors() & kv.LS_DEVERR_LENGTH
    c.dctx.copy_(i32_dev([2**31 - 10, 50]))
    c.run("device")
    assert kv.ls_device_errors() & kv.LS_DEVERR_LENGTH
    c.dctx.copy_(i32_dev(c.c))
    keep = c.tables.clone()
    c.tables[0, 110 // BLOCK] = -2
    for mode in ("device", "full"):
        c.run(mode)                                  # an id outside the pool: its keys are absent
    kv.ls_device_errors()
    c.tables.copy_(keep)
    c.check(what="afterwards")
