"""Sessions for the tests of shared prefixes, accumulated weights and eviction: pools in which slots
without a token are poisoned, the operators in 64 bits, and the bounds that results are held to."""
import numpy as np
import torch

from paper_2606_22983_amd import workloads as W
from tests.gpu_util import bf16_dev, i32_dev

BLOCK = 16


class Cache:
    """lens[s] tokens per session at shuffled blocks; the sessions of groups[g] = (members, blocks) have their
    first blocks in common (a member may be shorter).  Slots without a token hold NaN, table entries of
    blocks without a token an id outside the pool."""

    def __init__(self, rng, lens, hkv, d, groups=(), layers=1, extra_cols=2, spare=5, key_scale=1.0):
        self.lens, self.hkv, self.d, self.layers = np.asarray(lens, dtype=np.int64), hkv, d, layers
        s = len(self.lens)
        need = -(-self.lens // BLOCK)
        cols = max(1, int(need.max(initial=0))) + extra_cols
        self.tables = np.full((s, cols), -9, dtype=np.int32)
        self.groups = [(list(m), int(p)) for m, p in groups]
        lead = {}
        for m, p in self.groups:
            longest = max(m, key=lambda x: self.lens[x])
            for x in m:
                lead[x] = (longest, p)
        nb = int(need.sum()) + spare
        perm, at = rng.permutation(nb).astype(np.int32), 0
        for i in sorted(range(s), key=lambda x: lead.get(x, (x, 0))[0] != x):      # (a group's longest member first)
            longest, p = lead.get(i, (i, 0))
            for j in range(int(need[i])):
                if longest != i and j < p:
                    self.tables[i, j] = self.tables[longest, j]
                else:
                    self.tables[i, j] = perm[at]
                    at += 1
        self.pool = np.full((layers, nb, 2, hkv, BLOCK * d), W.NAN_BF16, dtype=np.uint16)
        for i in sorted(range(s), key=lambda x: self.lens[x]):
            t = np.arange(self.lens[i])
            for layer in range(layers):
                k = rng.standard_normal((len(t), hkv, d), dtype=np.float32) * key_scale
                self.write(layer, i, t, W.to_bf16(k), W.normal_bf16(rng, (len(t), hkv, d)))

    def write(self, layer, s, t, k, v):
        """Rows k, v [n][hkv][d] (bf16 bits) to tokens t of a session."""
        nb, hkv, d = self.pool.shape[1], self.hkv, self.d
        b, o = self.tables[s, t // BLOCK], t % BLOCK
        kt = self.pool[layer, :, 0].reshape(nb, hkv, d // 8, BLOCK, 8)
        vt = self.pool[layer, :, 1].reshape(nb, hkv, d, BLOCK)
        kt[b, :, :, o] = k.reshape(len(t), hkv, d // 8, 8)
        vt[b, :, :, o] = v
        assert np.shares_memory(kt, self.pool) and np.shares_memory(vt, self.pool)

    def rows(self, layer, s, t):
        """K and V of tokens t in 64 bits, [n][hkv][d]."""
        return rows_of(self.pool[layer], self.tables[s], t, self.d)

    def device(self, kv):
        self.data = bf16_dev(self.pool)
        self.dtables = i32_dev(self.tables)
        return kv.kv_pool_create(self.data, self.layers, self.pool.shape[1], self.hkv, self.d)

    def group_arrays(self):
        """(starts, members, prefix) on the device, or three Nones."""
        if not self.groups:
            return None, None, None
        members = [x for m, _ in self.groups for x in m]
        return (i32_dev(np.cumsum([0] + [len(m) for m, _ in self.groups])), i32_dev(members),
                i32_dev([p for _, p in self.groups]))

    def prefix_of(self, s):
        """Tokens of the session that its group shares."""
        return next((p * BLOCK for m, p in self.groups if s in m), 0)

    def entries(self, rng):
        """Weights and positions of every slot."""
        shape = (self.layers, self.pool.shape[1], self.hkv, BLOCK)
        return (np.exp(rng.standard_normal(shape)).astype(np.float32),
                rng.integers(-1000, 1000, shape, dtype=np.int32))


def rows_of(pool, table, t, d):
    """K and V of tokens t of a table row, [n][hkv][d] in 64 bits; pool: one layer's bits."""
    nb, _, hkv, _ = pool.shape
    b, o = table[t // BLOCK], t % BLOCK
    k = pool[:, 0].reshape(nb, hkv, d // 8, BLOCK, 8)[b, :, :, o].reshape(len(t), hkv, d)
    v = pool[:, 1].reshape(nb, hkv, d, BLOCK)[b, :, :, o]
    return W.from_bf16(k).astype(np.float64), W.from_bf16(v).astype(np.float64)


def attend(q, k, v, seen, scale):
    """q [R][hq][d] over k, v [n][hkv][d] with the mask seen [R][n], in 64 bits.  Returns out [R][hq][d], mass =
    sum p |v|, the largest sum of sizes of a score's products [R][hq], p [R][hq][n]."""
    r, hq, d = q.shape
    n, hkv = k.shape[:2]
    g = hq // hkv
    qg = q.reshape(r, hkv, g, d)
    x = np.einsum("rhgd,nhd->rhgn", qg, k) * scale
    size = np.einsum("rhgd,nhd->rhgn", np.abs(qg), np.abs(k)) * scale
    x = np.where(seen[:, None, None], x, -np.inf)
    with np.errstate(invalid="ignore"):
        p = np.exp(x - x.max(-1, keepdims=True, initial=-1e300))
    p /= np.maximum(p.sum(-1, keepdims=True), 1e-300)
    out = np.einsum("rhgn,nhd->rhgd", p, v).reshape(r, hq, d)
    mass = np.einsum("rhgn,nhd->rhgd", p, np.abs(v)).reshape(r, hq, d)
    score = np.where(seen[:, None, None], size, 0).max(-1, initial=0).reshape(r, hq)
    return out, mass, score, p.reshape(r, hq, n)


def decode_reference(c, layer, q, scale):
    """Every session's step in 64 bits: out, mass, score and a list of p [hq][L]."""
    outs, masses, scores, ps = [], [], [], []
    for s, n in enumerate(c.lens):
        k, v = c.rows(layer, s, np.arange(n))
        o, m, sc, p = attend(W.from_bf16(q[s:s + 1]).astype(np.float64), k, v, np.ones((1, n), dtype=bool), scale)
        outs.append(o[0])
        masses.append(m[0])
        scores.append(sc[0])
        ps.append(p[0])
    return np.stack(outs), np.stack(masses), np.stack(scores), ps


def weight_bound(p, score, d):
    """How far the sum over rows of p [R][G][n] may be off, [n]; score [R][G].

    p = 2^(x - m) / l.  As for an output: a score's fp32 sum of d products is off by (d - 1) 2^-24 of the sum of
    their sizes, scaling, maximum and the row's own logarithm by a rounding each of values of that size:
    (d + 6) 2^-23 score in the exponent, in numerator and sum.  exp2, division and the fp32 sums: 2^-12."""
    e = 2 * (d + 6) * 2.0 ** -23 * score[..., None] + 2.0 ** -12
    return (e * p).sum((0, 1))


def assert_entries(got, ref, tol, what):
    """Weights within their bounds; entries whose bound is 0 are to be the same bits."""
    g = got.cpu().numpy()
    err = np.abs(g.astype(np.float64) - ref)
    ok = err <= tol
    assert ok.all(), "%s: %d entries off, worst %.3e over %.3e" % (
        what, int((~ok).sum()), float(err[~ok].max()), float(tol[~ok][np.argmax(err[~ok])]))
    used = tol > 0
    if used.any():
        print("%s: worst err / bound %.3f (%d entries)" % (what, float((err[used] / tol[used]).max()), int(used.sum())),
              flush=True)


def add_weights(c, layer, s, sums, tol, w, pos, bound, first, old, begin):
    """Adds sums [hkv][n] to the reference's entries w, pos (64-bit and int32 arrays of all layers) of session s."""
    n = sums.shape[1]
    for t in range(first, n):
        b, o = c.tables[s, t // BLOCK], t % BLOCK
        if t >= old:
            w[layer, b, :, o] = sums[:, t]
            pos[layer, b, :, o] = begin + t - old
        else:
            w[layer, b, :, o] += sums[:, t]
        # (the sum's own rounding, and that of what was there)
        bound[layer, b, :, o] += tol[:, t] + 2.0 ** -23 * np.abs(w[layer, b, :, o])


def evict_reference(pool, tables, lens, budget, limit, recent, first, next_pos, w, pos, layers, d):
    """kv_evict on the host, slot by slot: pool, weights and positions after it (copies), and lengths."""
    pool, wn, pn = pool.copy(), w.copy(), pos.copy()
    keep = []
    nb, hkv = pool.shape[1], pool.shape[3]
    for s, n in enumerate(lens):
        m = int(n)
        if n > limit:
            m = min(int(n), max(budget, int(first[s]) + recent))
        keep.append(m)
        if m >= n:
            continue
        t = np.arange(n)
        b, o = tables[s, t // BLOCK], t % BLOCK
        for layer in layers:
            kt = pool[layer, :, 0].reshape(nb, hkv, d // 8, BLOCK, 8)
            vt = pool[layer, :, 1].reshape(nb, hkv, d, BLOCK)
            for h in range(hkv):
                ws, ps = w[layer, b, h, o], pos[layer, b, h, o]

                def rank(i):                      # best first
                    if i < first[s]:
                        return (0, 0.0, i)
                    if ps[i] >= next_pos[s] - recent:
                        return (1, 0.0, i)
                    return (2, np.inf if np.isnan(ws[i]) else -float(ws[i]), i) if not np.isnan(ws[i]) else (3, 0.0, i)
                stay = set(sorted(range(n), key=rank)[:m])
                src = sorted(i for i in stay if i >= m)
                dst = sorted(set(range(m)) - stay)
                assert len(src) == len(dst)
                for x, y in zip(src, dst):
                    kt[b[y], h, :, o[y]] = kt[b[x], h, :, o[x]]
                    vt[b[y], h, :, o[y]] = vt[b[x], h, :, o[x]]
                    wn[layer, b[y], h, o[y]] = ws[x]
                    pn[layer, b[y], h, o[y]] = ps[x]
    return pool, wn, pn, np.asarray(keep, dtype=np.int32)


def bits(t: torch.Tensor):
    return t.view(torch.int16).cpu().numpy().view(np.uint16)
