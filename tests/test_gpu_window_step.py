"""Windowed serving as a program runs it: tables from lengths, rows into their slots, attention over
what the window shows, blocks behind it used again by other sessions, the decode loop as one graph."""
import numpy as np
import pytest
import torch

from paper_2606_22983_amd import workloads as W
from tests.gpu_util import bf16_dev, i32_dev
from tests.window_util import BLOCK, assert_within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    from paper_2606_22983_amd import kv as kv_mod
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return kv_mod


class History:
    """Every session's K and V rows in logical order, and the reference over them."""

    def __init__(self, sessions, hkv, d):
        self.k = [np.empty((0, hkv, d), dtype=np.uint16) for _ in range(sessions)]
        self.v = [np.empty((0, hkv, d), dtype=np.uint16) for _ in range(sessions)]
        self.hkv, self.d = hkv, d

    def add(self, s, k, v):
        self.k[s], self.v[s] = np.concatenate([self.k[s], k]), np.concatenate([self.v[s], v])

    def reference(self, oracle, q, who, pos, scale, window, sinks):
        need = [(len(k) + 15) // 16 for k in self.k]
        pool = np.full((1, max(1, sum(need)), 2, self.hkv, 16 * self.d), W.NAN_BF16, dtype=np.uint16)
        tables = np.zeros((len(need), max(need)), dtype=np.int32)
        at = 0
        for s, n in enumerate(need):
            tables[s, :n] = np.arange(at, at + n)
            at += n
            oracle.append(pool, 16, self.d, 0, tables, np.full(len(self.k[s]), s), np.arange(len(self.k[s])), self.k[s], self.v[s])
        return oracle.attend_window(pool, 16, self.d, 0, q, tables, who, pos, np.arange(len(who)), scale, window, sinks)


def test_turns_and_a_captured_decode_loop(kv, oracle_lib):
    S, hq, hkv, d, window, sinks, layers = 6, 16, 2, 64, 50, 4, 2
    cols, nb = 40, 60                                     # fewer blocks than the histories have in the end
    rng = np.random.default_rng(1)
    scale = d ** -0.5
    data = torch.full((layers, nb, 2, hkv, 16 * d), float("nan"), dtype=torch.bfloat16, device="cuda")
    pool = kv.kv_pool_create(data, layers, nb, hkv, d)
    tables = torch.full((S, cols), -1, dtype=torch.int32, device="cuda")
    lens, reused = torch.zeros(S, dtype=torch.int32, device="cuda"), torch.zeros(S, dtype=torch.int32, device="cuda")
    ring = torch.full((2 * nb,), -1, dtype=torch.int32, device="cuda")          # turns may be longer than the window
    ring[:nb] = torch.from_numpy(rng.permutation(nb).astype(np.int32)).cuda()
    counts = torch.tensor([0, nb], dtype=torch.int64, device="cuda")
    cu = torch.zeros(S + 1, dtype=torch.int32, device="cuda")
    hist = [History(S, hkv, d) for _ in range(layers)]
    host_lens = np.zeros(S, dtype=np.int64)

    def turn(n):
        """One batched turn of n[s] new tokens."""
        total, pad = int(sum(n)), 5
        slots = torch.empty(total + pad, dtype=torch.int64, device="cuda")
        kv.kv_tables_update(pool, lens, i32_dev(n), int(max(n)), tables, lens, cu, reused, slots, free_ring=ring,
                            free_counts=counts, next_counts=counts, window=window, sinks=sinks)
        who = np.repeat(np.arange(S), n)
        pos = np.concatenate([np.arange(host_lens[s], host_lens[s] + n[s]) for s in range(S)]).astype(np.int32)
        outs = []
        for layer in range(layers):
            qkv = W.normal_bf16(rng, (total + pad, hq + 2 * hkv, d))
            dev = bf16_dev(qkv)
            kv.kv_append(pool, layer, dev[:, hq:hq + hkv], dev[:, hq + hkv:], slots)
            q = dev[:, :hq].contiguous()
            out = torch.full_like(q, 3.0)
            kv.paged_attn_prefill_window(pool, layer, q, cu, reused, int(max(n)), tables, window, sinks, scale, out)
            for s in range(S):
                m = np.nonzero(who == s)[0]
                hist[layer].add(s, qkv[m, hq:hq + hkv], qkv[m, hq + hkv:])
            outs.append((out, qkv[:, :hq]))
        host_lens[:] += n
        torch.cuda.synchronize()
        assert kv.ls_device_errors() == 0
        for layer, (out, q) in enumerate(outs):
            ref = hist[layer].reference(oracle_lib, q[:total], who, pos, scale, window, sinks)
            assert_within(out[:total], *ref, d, "turn, layer %d" % layer)
            assert (out[total:] == 3.0).all()

    turn([40, 1, 17, 0, 90, 16])
    turn([0, 30, 1, 70, 3, 16])

    # the decode loop: lengths, tables and counters advance on the GPU, nothing comes from the host
    ones = torch.ones(S, dtype=torch.int32, device="cuda")
    slots = torch.empty(S, dtype=torch.int64, device="cuda")
    q, out = (torch.empty((layers, S, hq, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kn, vn = (torch.empty((layers, S, hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ws = torch.empty(kv.decode_window_workspace_bytes(pool, S, hq, cols, window, sinks), dtype=torch.uint8, device="cuda")

    def step():
        kv.kv_tables_update(pool, lens, ones, 1, tables, lens, cu, reused, slots, free_ring=ring, free_counts=counts,
                            next_counts=counts, window=window, sinks=sinks)
        for layer in range(layers):
            kv.paged_attn_decode_window(pool, layer, q[layer], tables, reused, window, sinks, scale, out[layer], ws, kn[layer],
                                        vn[layer])

    def inputs():
        x = [W.normal_bf16(rng, (layers, S, h, d)) for h in (hq, hkv, hkv)]
        for t, a in zip((q, kn, vn), x):
            t.copy_(bf16_dev(a))
        for layer in range(layers):
            for s in range(S):
                hist[layer].add(s, x[1][layer, s:s + 1], x[2][layer, s:s + 1])
        return x[0]

    def compare(hq_bits, what):
        torch.cuda.synchronize()
        host_lens[:] += 1
        assert kv.ls_device_errors() == 0, what
        for layer in range(layers):
            ref = hist[layer].reference(oracle_lib, hq_bits[layer], np.arange(S), host_lens - 1, scale, window, sinks)
            assert_within(out[layer], *ref, d, what)

    bits = inputs()
    step()
    compare(bits, "eager step")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(150):
        bits = inputs()
        graph.replay()
        if i % 10 == 9:
            compare(bits, "step %d" % i)
        else:
            host_lens[:] += 1
    total_blocks = int(((host_lens + 15) // 16).sum())
    assert total_blocks > nb                              # the pool could not have held the histories
    assert int(lens.sum()) == int(host_lens.sum())
    turn([5, 60, 0, 33, 1, 2])                            # a turn after the loop
    free = ring.cpu().numpy()[(np.arange(int(counts[0]), int(counts[1]))) % (2 * nb)]
    assert len(set(free.tolist())) == len(free)           # no block is free twice


def test_calls_at_once_on_three_streams(kv, oracle_lib):
    """A decode, a prefill and an append over disjoint blocks of one pool, with scratch of their own, in flight together."""
    hq, hkv, d, window, sinks = 16, 4, 128, 300, 20
    rng = np.random.default_rng(2)
    scale = d ** -0.5
    lens, n, c = np.array([900, 70, 2000, 333], dtype=np.int32), np.array([130, 1, 500], dtype=np.int32), np.array([700, 40, 0], dtype=np.int32)
    have = np.concatenate([lens, c])
    need = -(-np.concatenate([lens, c + n]) // BLOCK)
    nb, cols = int(need.sum()) + 40, int(need.max())
    tables = np.zeros((len(need), cols), dtype=np.int32)
    ids, at = rng.permutation(nb), 0
    for s, k in enumerate(need):
        tables[s, :k] = ids[at:at + k]
        at += k
    host = np.full((1, nb, 2, hkv, BLOCK * d), W.NAN_BF16, dtype=np.uint16)
    for s, k in enumerate(have):
        kv_rows = [W.normal_bf16(rng, (k, hkv, d)) for _ in range(2)]
        oracle_lib.append(host, BLOCK, d, 0, tables, np.full(k, s), np.arange(k), *kv_rows)
    data = bf16_dev(host)
    pool = kv.kv_pool_create(data, 1, nb, hkv, d)
    T = int(n.sum())
    dq, pq, pk, pv = (W.normal_bf16(rng, (r, h, d)) for r, h in ((4, hq), (T, hq), (T, hkv), (T, hkv)))
    ak, av = (W.normal_bf16(rng, (40 * BLOCK, hkv, d)) for _ in range(2))
    slots = (ids[at:at + 40, None] * BLOCK + np.arange(BLOCK)).reshape(-1)
    dev = [bf16_dev(x) for x in (dq, pq, pk, pv, ak, av)]
    dtab, ptab = i32_dev(tables[:4]), i32_dev(tables[4:])
    dl, pc, cu = i32_dev(lens), i32_dev(c), i32_dev(np.concatenate([[0], np.cumsum(n)]))
    dout, pout = (torch.full_like(x, float("nan")) for x in dev[:2])
    ws = torch.empty(kv.decode_window_workspace_bytes(pool, 4, hq, cols, window, sinks), dtype=torch.uint8, device="cuda")
    pws = torch.empty(kv.PREFILL_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    dslots = torch.from_numpy(slots.astype(np.int64)).cuda()
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(5):
        kv.paged_attn_prefill_window(pool, 0, dev[1], cu, pc, int(n.max()), ptab, window, sinks, scale, pout, dev[2], dev[3],
                                     lens_host=np.stack([n, c], 1), workspace=pws, stream=streams[0])
        kv.paged_attn_decode_window(pool, 0, dev[0], dtab, dl, window, sinks, scale, dout, ws, context_lens_host=lens, stream=streams[1])
        kv.kv_append(pool, 0, dev[4], dev[5], dslots, stream=streams[2])
    torch.cuda.synchronize()
    assert kv.ls_device_errors() == 0
    who = np.repeat(np.arange(3), n) + 4
    pos = np.concatenate([np.arange(a, a + b) for a, b in zip(c, n)]).astype(np.int32)
    oracle_lib.append(host, BLOCK, d, 0, tables, who, pos, pk, pv)
    oracle_lib.append_slots(host, BLOCK, d, 0, ak, av, slots)
    assert np.array_equal(data.view(torch.int16).cpu().numpy().view(np.uint16).reshape(host.shape), host)
    assert_within(pout, *oracle_lib.attend_window(host, BLOCK, d, 0, pq, tables, who, pos, np.arange(T), scale, window, sinks), d, "prefill")
    assert_within(dout, *oracle_lib.attend_window(host, BLOCK, d, 0, dq, tables, np.arange(4), lens - 1, np.arange(4), scale, window,
                                                  sinks), d, "decode")


def test_nothing_to_do(kv, oracle_lib):
    """No sessions, no tokens, one row of a wider tensor."""
    data = torch.zeros((1, 4, 2, 2, 16 * 64), dtype=torch.bfloat16, device="cuda")
    pool = kv.kv_pool_create(data, 1, 4, 2, 64)
    i32 = dict(dtype=torch.int32, device="cuda")
    none, tables = torch.empty(0, **i32), torch.empty((0, 3), **i32)
    cu, slots = torch.full((1,), 9, **i32), torch.full((3,), 9, dtype=torch.int64, device="cuda")
    ring, counts = torch.zeros(8, **i32), torch.tensor([3, 7], dtype=torch.int64, device="cuda")
    after = torch.zeros_like(counts)
    kv.kv_tables_update(pool, none, none, 0, tables, none, cu, none, slots, ring, counts, after, 16, 0)
    assert cu.tolist() == [0] and slots.tolist() == [-1, -1, -1] and after.tolist() == [3, 7]
    lens, new = torch.tensor([5, 0], **i32), torch.zeros(2, **i32)
    tables, nxt, cu = torch.full((2, 3), 1, **i32), torch.empty(2, **i32), torch.empty(3, **i32)
    kv.kv_tables_update(pool, lens, new, 0, tables, nxt, cu, None, slots[:0], ring, counts, after, 16, 0)
    assert nxt.tolist() == [5, 0] and cu.tolist() == [0, 0, 0] and after.tolist() == [3, 7] and (tables == 1).all()
    rows = torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    kv.kv_append(pool, 0, rows, rows, slots[:0])
    assert (data == 0).all()
    wide = torch.ones((1, 9, 64), dtype=torch.bfloat16, device="cuda")
    kv.kv_append(pool, 0, wide[:, 2:4], wide[:, 6:8], torch.tensor([37], device="cuda"))
    assert int((data != 0).sum()) == 2 * 2 * 64
    q = torch.empty((0, 8, 64), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(4096, dtype=torch.uint8, device="cuda")
    kv.paged_attn_decode_window(pool, 0, q, tables[:0], lens[:0], 16, 0, 0.125, torch.empty_like(q), ws)
    kv.paged_attn_prefill_window(pool, 0, q, torch.zeros(1, **i32), lens[:0], 0, tables[:0], 16, 0, 0.125, torch.empty_like(q))
    assert kv.ls_device_errors() == 0
