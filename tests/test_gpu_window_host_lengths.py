"""paged_attn_decode_window with host lengths that differ from the device's: a captured step that is
replayed while the lengths on the GPU advance."""
import numpy as np
import pytest
import torch

from tests.gpu_util import host_bits, i32_dev
from tests.test_gpu_window_decode import Case as Decode
from tests.window_util import assert_within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    from paper_2606_22983_amd import kv as kv_mod
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return kv_mod


@pytest.mark.parametrize("window,host", [(512, 600), (512, 1000), (1024, 1500), (700, 720)])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64), (32, 4, 128)])
@pytest.mark.parametrize("delta", [-40, -16, -9, -1, 1, 16, 23, 40])
def test_lagging_host_lengths_never_write_another_slot(kv, oracle_lib, window, host, hq, hkv, d, delta):
    """The step's row goes to its own slot or nowhere, though every other column names a block; and a
    plan that still covers the device's lengths gives their result."""
    lens = [host + delta, host, host - delta]
    c = Decode(kv, oracle_lib, lens, window, 4, hq, hkv, d, True, seed=window + delta)
    tables = c.ses.tables
    nb = c.ses.pool.shape[1]
    named = (tables >= 0) & (tables < nb)
    spare = np.setdiff1d(np.arange(nb), tables[named])
    tables[~named] = np.resize(spare, int((~named).sum()))
    c.tables.copy_(i32_dev(tables))
    before = host_bits(c.data).reshape(c.ses.pool.shape).copy()
    work, (ref, mass, score) = c.reference()
    out = c.run(True, lens_host=np.full(3, host, dtype=np.int32))
    bits = kv.ls_device_errors()
    assert bits in (0, kv.LS_DEVERR_LENGTH)
    got = host_bits(c.data).reshape(before.shape)
    if bits == 0:
        assert np.array_equal(got, work)
        assert_within(out, ref, mass, score, d, "host %d device %s" % (host, lens))
    else:                                             # a session past its plan: its row may be missing
        for a, b in ((0, 0), (0, 1)):
            g, x, y = (p[a, :, b] for p in (got, before, work))
            assert ((g == x) | (g == y)).all()
