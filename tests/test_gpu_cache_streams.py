"""Weights of turns and evictions in captured graphs, on two streams at once, and on streams of few CUs."""
import numpy as np
import pytest
import torch

from paper_2606_22983_amd import workloads as W
from tests.cache_util import BLOCK, Cache
from tests.gpu_util import bf16_dev, cu_masked_stream, destroy_stream, i32_dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    from paper_2606_22983_amd import kv as kv_mod
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    kv_mod.ls_device_errors()
    return kv_mod


class Turn:
    """A call of kv_weights_prefill with a workspace of its own, from zero weights."""

    def __init__(self, kv, seed, lens, n, rows, hkv, hq, d, layers=1, layer=0, shared=None):
        rng = np.random.default_rng(seed)
        self.kv, self.c, self.layer, self.rows, self.d = kv, shared or Cache(rng, lens, hkv, d, layers=layers), layer, rows, d
        self.pool = self.c.device(kv) if shared is None else None
        s, self.n = len(lens), n
        self.q = bf16_dev(W.normal_bf16(rng, (s * n, hq, d)))
        self.cu, self.ctx = i32_dev(np.arange(s + 1) * n), i32_dev(self.c.lens - n)
        shape = (layers, self.c.pool.shape[1], hkv, BLOCK)
        self.w, self.p = torch.zeros(shape, device="cuda"), torch.zeros(shape, dtype=torch.int32, device="cuda")

    def workspace(self, pool):
        hq = self.q.shape[1]
        size = self.kv.weights_prefill_workspace_bytes(pool, len(self.c.lens), hq, self.q.shape[0], self.n, self.rows, self.c.tables.shape[1])
        self.pool, self.ws = pool, torch.full((size,), 255, dtype=torch.uint8, device="cuda")
        return self

    def __call__(self, stream=None):
        self.kv.kv_weights_prefill(self.pool, self.layer, self.q, self.cu, self.ctx, self.n, self.c.dtables, self.rows, self.d ** -0.5,
                                   self.w, self.p, self.ws, stream=stream)


def test_captured_turns(kv):
    """Rows of three rounds; lengths that change between replays, and the caller's own work between them."""
    t = Turn(kv, 1, [500, 420], 300, 300, 2, 16, 128)
    t.workspace(t.pool)
    full = t.ctx.clone()
    t()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        t()
    for less in (0, 17, 100, 0):
        t.ctx.copy_(full - less)
        t.w.fill_(0.5)
        t.p.zero_()
        t()
        torch.cuda.synchronize()
        want = t.w.clone(), t.p.clone()
        t.w.fill_(0.5)
        t.p.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(t.w, want[0]) and torch.equal(t.p, want[1])
    assert kv.ls_device_errors() == 0


def test_turns_at_once(kv):
    """Two layers of one pool, each on a stream and with weights and a workspace of its own."""
    a = Turn(kv, 2, [900, 3000, 64], 60, 40, 4, 32, 128, layers=2)
    b = Turn(kv, 3, [900, 3000, 64], 60, 60, 4, 32, 128, layers=2, layer=1, shared=a.c)
    a.workspace(a.pool)
    b.workspace(a.pool)
    alone = []
    for t in (a, b):
        for _ in range(10):
            t()
        torch.cuda.synchronize()
        alone.append((t.w.clone(), t.p.clone()))
        t.w.zero_()
        t.p.zero_()
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for t, st in zip((a, b), streams):
            t(st)
    torch.cuda.synchronize()
    assert kv.ls_device_errors() == 0
    for t, (w, p) in zip((a, b), alone):
        assert torch.equal(t.w, w) and torch.equal(t.p, p)


@pytest.mark.parametrize("cus", [8, 40])
def test_on_a_stream_of_few_cus(kv, cus):
    """A turn's weights and an eviction give the same bits, a decode with weights the same within its rounding."""
    rng = np.random.default_rng(4)
    c = Cache(rng, [700, 350, 1200, 90], 2, 64)
    pool = c.device(kv)
    made = cu_masked_stream(0, cus)
    if made is None:
        pytest.skip("no stream with a CU mask")
    stream, handle = made
    t = Turn(kv, 5, c.lens, 30, 30, 2, 8, 64, shared=c).workspace(pool)
    q, lens = bf16_dev(W.normal_bf16(rng, (4, 8, 64))), i32_dev(c.lens)
    ws = torch.full((kv.decode_weights_workspace_bytes(pool, 4, 8),), 255, dtype=torch.uint8, device="cuda")
    out, nxt = torch.empty_like(q), torch.empty_like(lens)
    after = i32_dev(c.lens)
    got = []
    for st in (None, stream):
        t.w.zero_()
        wn, pn, w2 = torch.zeros_like(t.w), torch.zeros_like(t.p), torch.zeros_like(t.w)
        c.data.copy_(bf16_dev(c.pool))
        torch.cuda.synchronize()
        t(st)
        kv.paged_attn_decode_weights(pool, 0, q, c.dtables, lens, 0.125, out, w2, None, ws, stream=st)
        kv.kv_evict(pool, lens, c.dtables, 300, 310, 50, after, t.w, t.p, nxt, wn, pn, stream=st)
        torch.cuda.synchronize()
        got.append([x.clone() for x in (t.w, t.p, wn, pn, nxt, c.data.view(torch.int16), w2)])
    destroy_stream(handle)
    assert kv.ls_device_errors() == 0
    for a, b in zip(got[0][:-1], got[1][:-1]):
        assert torch.equal(a, b)
    # two decodes, each off by 2^-12 and its scores' errors at most (64 products of size 3: 2 (64 + 6) 2^-23 of 20)
    a, b = got[0][-1].double(), got[1][-1].double()
    assert ((a - b).abs() <= 2 * (2.0 ** -12 + 2 * 70 * 2.0 ** -23 * 20) * torch.maximum(a, b)).all()
