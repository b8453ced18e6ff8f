"""paged_attn_decode_window with the least workspace it takes: no room for the single-launch kernel's
counts and partial results, so the persistent kernel runs, with its merge where a walk is split."""
import ctypes

import numpy as np
import pytest
import torch

from tests.gpu_util import host_bits
from tests.test_gpu_window_decode import Case
from tests.window_util import assert_within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    from paper_2606_22983_amd import kv as kv_mod
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return kv_mod


def split_tokens(kv, c, host, size):
    """Tokens per split of the single-launch kernel with a workspace of `size` bytes, 0: the persistent one."""
    lens = np.ascontiguousarray(c.lens, dtype=np.int32)
    t = kv.raw_library().ls_internal_small_decode_window(
        c.pool.handle, len(lens), c.q.shape[1], c.tables.shape[1], c.window, c.sinks,
        lens.ctypes.data_as(ctypes.c_void_p) if host else None, int(c.kn is not None), ctypes.c_void_p(c.ws.data_ptr()),
        ctypes.c_size_t(size), None)
    assert t >= 0
    return t


def least(kv, c):
    """The fewest bytes that a call takes."""
    lo, hi = 0, c.ws.numel()                          # refused, taken
    while hi - lo > 1:
        mid = (lo + hi) // 2
        try:
            c.run(False, workspace=c.ws[:mid])
            hi = mid
        except kv.LiveServeError as e:
            assert e.status == kv.LS_ENOMEM
            lo = mid
    return hi


@pytest.mark.parametrize("lens,window,sinks,hq,hkv,d,append", [
    # (every walk as long as a walk gets: with host lengths, the room that shorter ones leave is used)
    ([3000, 4000, 5000, 2222], 1200, 4, 16, 4, 128, True), ([9000, 3001, 2500], 1024, 20, 8, 2, 64, False),
    ([7000, 1300, 6000, 9000, 4900], 1230, 0, 8, 4, 64, True)])
def test_least_workspace(kv, oracle_lib, lens, window, sinks, hq, hkv, d, append):
    c = Case(kv, oracle_lib, lens, window, sinks, hq, hkv, d, append, seed=window)
    work, (ref, mass, score) = c.reference()
    size = least(kv, c)
    assert kv.ls_device_errors() == 0 and 0 < size < c.ws.numel()
    for host in (False, True):
        assert split_tokens(kv, c, host, c.ws.numel()) > 0 and split_tokens(kv, c, host, size) == 0
        behind = c.ws[size:].clone()
        for _ in range(2):
            c.ws[:size].random_()
            out = c.run(host, workspace=c.ws[:size])
            assert kv.ls_device_errors() == 0
            assert_within(out, ref, mass, score, d, "%d bytes, host lengths %s" % (size, host))
        assert torch.equal(c.ws[size:], behind)
    assert np.array_equal(host_bits(c.data).reshape(work.shape), work)
