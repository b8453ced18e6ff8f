"""Windowed prefill with host lengths and a workspace: a call whose items all have a CU of their own takes
them by index, so it neither needs the item counters nor pays the launch that clears them."""
import numpy as np
import pytest
import torch

from tests.test_gpu_window_prefill import Case
from tests.window_util import assert_within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    from paper_2606_22983_amd import kv as kv_mod
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return kv_mod


@pytest.mark.parametrize("turns,full,untouched", [
    ([(40, 300), (70, 20)], False, True), ([(301, 3000)], True, True), ([(301, 3000)], False, True),
    ([(300, 200)] * 30, False, False), ([(300, 200)] * 30, True, False)])       # (1200 items and more; 240 pairs, which a host plan holds)
@pytest.mark.parametrize("hq,hkv,d", [(16, 2, 64), (8, 2, 128)])
def test_turns_in_the_pool(kv, oracle_lib, turns, full, untouched, hq, hkv, d):
    c = Case(kv, oracle_lib, turns, 200, 4, 4 * hq, 4 * hkv, d, False, seed=d)
    rows = np.unique(np.concatenate([c.cu[:-1], c.cu[1:] - 1, np.arange(0, c.cu[-1], 97)]))
    _, ref = c.reference(rows)
    ws = c.ws if full else c.ws[:kv.PREFILL_COUNTER_BYTES]
    for _ in range(2):
        ws.fill_(0xAB)
        out = torch.full(c.q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
        kv.paged_attn_prefill_window(c.pool, 0, c.dq, c.dcu, c.dctx, int(c.n.max()), c.tables, 200, 4, c.scale, out,
                                     lens_host=c.lens_host, workspace=ws)
        torch.cuda.synchronize()
        assert kv.ls_device_errors() == 0
        assert_within(out[torch.from_numpy(rows).cuda()], *ref, d, "%d turns" % len(turns))
        assert bool((ws[:kv.PREFILL_COUNTER_BYTES] == 0xAB).all()) == untouched
