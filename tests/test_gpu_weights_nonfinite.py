"""A turn's weights where a query row is not a number: the keys that it sees get no number, the others the other rows' sums."""
import numpy as np
import pytest
import torch

from paper_2606_22983_amd import workloads as W
from tests.cache_util import BLOCK, Cache, attend, weight_bound
from tests.gpu_util import bf16_dev, i32_dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    from paper_2606_22983_amd import kv as kv_mod
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    kv_mod.ls_device_errors()
    return kv_mod


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("d,hkv,g,sessions,ctx,n,rows", [
    (128, 2, 4, 1, 0, 90, 1000), (128, 1, 8, 2, 37, 70, 40), (64, 2, 1, 1, 0, 300, 300), (64, 4, 2, 9, 3000, 40, 32),
    (64, 8, 1, 40, 700, 100, 100), (128, 1, 8, 1, 0, 300, 300)])
def test_keys_behind_the_row(kv, value, d, hkv, g, sessions, ctx, n, rows):
    rng = np.random.default_rng(n)
    c = Cache(rng, [ctx + n] * sessions, hkv, d)
    total, hq = sessions * n, hkv * g
    q = W.normal_bf16(rng, (total, hq, d))
    j, head = n - min(n, rows) + 5, hq - 1               # the sixth observed row of every turn, in one head
    q[j::n, head] = W.to_bf16(np.full(d, value, dtype=np.float32))
    pool = c.device(kv)
    shape = (1, c.pool.shape[1], hkv, BLOCK)
    weights, positions = torch.zeros(shape, device="cuda"), torch.zeros(shape, dtype=torch.int32, device="cuda")
    ws = torch.empty(kv.weights_prefill_workspace_bytes(pool, sessions, hq, total, n, rows, c.tables.shape[1]), dtype=torch.uint8,
                     device="cuda")
    kv.kv_weights_prefill(pool, 0, bf16_dev(q), i32_dev(np.arange(sessions + 1) * n), i32_dev([ctx] * sessions), n, c.dtables, rows,
                          d ** -0.5, weights, positions, ws)
    assert kv.ls_device_errors() == 0
    got = weights.cpu().numpy()[0]
    for s in range(min(sessions, 3)):
        t = np.arange(ctx + n)
        k, v = c.rows(0, s, t)
        obs = np.arange(max(0, n - rows), n)
        x = W.from_bf16(q[s * n + obs]).astype(np.float64)
        x[obs == j, head] = 0.0                          # (its row is left out of the sums below)
        _, _, score, p = attend(x, k, v, t[None] <= (ctx + obs)[:, None], d ** -0.5)
        p, score = p.reshape(len(obs), hkv, g, -1), score.reshape(len(obs), hkv, g)
        p[obs == j, hkv - 1, g - 1] = 0.0
        ref = p.sum((0, 2))
        tol = np.stack([weight_bound(p[:, h], score[:, h], d) for h in range(hkv)]) + 2.0 ** -12 * ref + 1e-30
        mine = got[c.tables[s, t // BLOCK], :, t % BLOCK].T
        seen = t <= ctx + j
        assert np.isnan(mine[hkv - 1, seen]).all()
        mine[hkv - 1, seen] = ref[hkv - 1, seen]
        err = np.abs(mine - ref)
        assert (err <= tol).all(), "session %d: %d keys off or not a number" % (s, int((~(err <= tol)).sum()))
