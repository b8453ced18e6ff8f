"""Windowed prefill: NaN and infinities in keys that no row of a query tile sees do not reach its rows.
(tests/test_gpu_window_prefill.py has them before the window and behind the turn; here they are the
turn's own later tokens.)"""
import numpy as np
import pytest
import torch

from tests.gpu_util import bf16_dev
from tests.test_gpu_window_prefill import Case
from tests.window_util import assert_within

pytestmark = pytest.mark.gpu

ROWS = 256                                            # (token, query head of a KV head) pairs of a query tile
NAN, INF, MINUS_INF = 0x7FC0, 0x7F80, 0xFF80


@pytest.fixture(scope="module")
def kv():
    from paper_2606_22983_amd import kv as kv_mod
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return kv_mod


def spoil(c, session, j, bits_k, bits_v):
    """K and V of the turn's token j: in the rows that the call appends, or in the pool."""
    p, hkv, d = int(c.c[session]) + j, c.ses.pool.shape[3], c.d
    if c.kn is not None:
        c.kn[c.cu[session] + j], c.vn[c.cu[session] + j] = bits_k, bits_v
    else:
        b, o = c.ses.tables[session, p // 16], p % 16
        c.ses.pool[c.layer, b, 0].reshape(hkv, d // 8, 16, 8)[:, :, o] = bits_k
        c.ses.pool[c.layer, b, 1].reshape(hkv, d, 16)[:, :, o] = bits_v


@pytest.mark.parametrize("turns,window,sinks", [
    ([(64, 0)], 64, 0), ([(300, 0)], 1000, 0), ([(70, 37), (290, 500)], 200, 9), ([(260, 1200), (40, 0)], 1 << 29, 0),
    ([(90, 3)], 5, 300), ([(513, 2500)], 2048, 4)])
@pytest.mark.parametrize("hq,hkv,d,append", [(8, 1, 64, True), (16, 2, 128, False), (2, 2, 128, True), (4, 2, 64, False)])
def test_later_tokens_of_the_turn(kv, oracle_lib, turns, window, sinks, hq, hkv, d, append):
    """The first token of some tile is spoilt: every tile before it gives what it gives without it."""
    c = Case(kv, oracle_lib, turns, window, sinks, hq, hkv, d, append, seed=window % 1000 + d)
    qtok = ROWS // (hq // hkv)
    rows = []
    for s, (n, _) in enumerate(turns):
        tile = -(-n // qtok) // 2                     # the tile from which on the rows may be spoilt
        j = tile * qtok if tile else n                # (a turn of one tile stays as it is)
        rows.append(int(c.cu[s]) + np.arange(j))
        if tile:
            spoil(c, s, j, NAN, (NAN, INF, MINUS_INF)[s % 3])
            if j + 1 < n:
                spoil(c, s, j + 1, INF, MINUS_INF)
    rows = np.concatenate(rows)
    c.data.copy_(bf16_dev(c.ses.pool))
    if append:
        c.dkn.copy_(bf16_dev(c.kn))
        c.dvn.copy_(bf16_dev(c.vn))
    _, (ref, mass, score) = c.reference(rows)
    assert np.isfinite(ref).all()
    for mode in ("device", "host", "counters", "full"):
        out = c.run(mode)
        assert kv.ls_device_errors() == 0
        assert_within(out[torch.from_numpy(rows).cuda()], ref, mass, score, d, "%s, spoilt from a tile on" % mode)
