"""Sessions for the tests of windowed attention: pools in which whatever a call must not use is
poisoned, and the error bound that its outputs are held to."""
import numpy as np

from paper_2606_22983_amd import workloads as W

BLOCK = 16
STALE = np.array([-1, -7, 2**31 - 1, 12345678], dtype=np.int32)     # table entries that a call must not read


def visible(p, t, window, sinks):
    return (t <= p) & ((t < sinks) | (t > p - window))


class Sessions:
    """``total[s]`` tokens per session at shuffled blocks; the rows of a call stand at positions
    first[s] .. last[s].  Tokens that no row sees hold NaN, and table entries of blocks that hold no
    token seen by a row hold ids outside the pool."""

    def __init__(self, rng, first, last, window, sinks, hkv, d, extra_cols=3, spare=5, layers=1, layer=0,
                 key_scale=None):
        first, last = np.asarray(first, dtype=np.int64), np.asarray(last, dtype=np.int64)
        s = len(first)
        cols = max(1, int((last.max() + BLOCK) // BLOCK)) + extra_cols
        self.tables = np.resize(STALE, (s, cols)).astype(np.int32).copy()
        seen_blocks = []
        for i in range(s):
            t = np.arange(last[i] + 1)
            seen = (t < sinks) | (t > first[i] - window)              # (a later row's window starts later)
            seen_blocks.append(np.unique(t[seen] // BLOCK))
        used = sum(len(b) for b in seen_blocks)
        nb = used + spare
        perm = rng.permutation(nb).astype(np.int32)
        self.pool = np.full((layers, nb, 2, hkv, BLOCK * d), W.NAN_BF16, dtype=np.uint16)
        kt = self.pool[layer, :, 0].reshape(nb, hkv, d // 8, BLOCK, 8)
        vt = self.pool[layer, :, 1].reshape(nb, hkv, d, BLOCK)
        at = 0
        for i in range(s):
            ids = perm[at:at + len(seen_blocks[i])]
            at += len(ids)
            self.tables[i, seen_blocks[i]] = ids
            t = np.arange(last[i] + 1)
            t = t[(t < sinks) | (t > first[i] - window)]
            k = rng.standard_normal((len(t), hkv, d), dtype=np.float32)
            if key_scale is not None:
                k *= key_scale(t, int(last[i]) + 1)[:, None, None].astype(np.float32)
            b, o = self.tables[i, t // BLOCK], t % BLOCK
            kt[b, :, :, o] = W.to_bf16(k).reshape(len(t), hkv, d // 8, 8)
            vt[b, :, :, o] = W.normal_bf16(rng, (len(t), hkv, d))

    def poison(self, layer, session, positions, d):
        """NaN into the K and V of some tokens of a session."""
        nb, hkv = self.pool.shape[1], self.pool.shape[3]
        kt = self.pool[layer, :, 0].reshape(nb, hkv, d // 8, BLOCK, 8)
        vt = self.pool[layer, :, 1].reshape(nb, hkv, d, BLOCK)
        t = np.asarray(positions)
        b, o = self.tables[session, t // BLOCK], t % BLOCK
        kt[b, :, :, o] = W.NAN_BF16
        vt[b, :, :, o] = W.NAN_BF16


def bound(ref, mass, score, d):
    """How far a bf16 output may be from the 64-bit one.

    o = sum p v / sum p.  Each p enters the numerator rounded to bf16 (2^-8 relative at most) and, in
    prefill, the sum as well: 2 * 2^-8 of mass = sum w |v|.  A score is an fp32 sum of d products, off
    by (d - 1) 2^-24 of the sum of their sizes, then scaled and shifted (one rounding each of values up
    to twice the largest score): (d + 4) 2^-23 score in the exponent, in numerator and sum.  exp2, the
    fp32 sums over keys (a few thousand, in partial sums of some hundred) and the division: 2^-12.  The
    result is rounded to bf16: 2^-8 of its own size, of which nothing is left out."""
    e = 2 * 2.0 ** -8 + 2 * (d + 4) * 2.0 ** -23 * score[..., None] + 2.0 ** -12
    return e * mass * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref)


def assert_within(gpu, ref, mass, score, d, what):
    g = gpu.float().cpu().numpy().astype(np.float64).reshape(ref.shape)
    assert np.isfinite(g).all(), "%s: non-finite output" % what
    err, tol = np.abs(g - ref), bound(ref, mass, score, d)
    rms = float(np.sqrt(np.mean(err ** 2)) / max(np.sqrt(np.mean(ref ** 2)), 1e-30))
    print("%s: worst err / bound %.3f, rms-rel %.2e (%d values)" % (what, float((err / tol).max()), rms, ref.size),
          flush=True)
    assert (err <= tol).all(), "%s: err %.3e over bound %.3e" % (what, float(err.max()),
                                                                float(tol.flat[np.argmax(err - tol)]))
