"""Decode with accumulated weights and groups that cannot be: outputs as without groups, weights and positions untouched."""
import numpy as np
import pytest
import torch

from paper_2606_22983_amd import workloads as W
from tests.cache_util import BLOCK, Cache, decode_reference
from tests.gpu_util import bf16_dev, i32_dev
from tests.window_util import assert_within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    from paper_2606_22983_amd import kv as kv_mod
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    kv_mod.ls_device_errors()
    return kv_mod


@pytest.mark.parametrize("sessions", [4, 520])                   # either schedule
@pytest.mark.parametrize("what", ["twice", "outside", "negative", "falling", "open start", "open end", "long prefix", "negative prefix"])
def test_entries_stay(kv, what, sessions):
    """The members have blocks in common whose scores are every member's: none of them is added up."""
    rng = np.random.default_rng(10)
    lens = np.concatenate([[100, 200, 300, 50], rng.integers(1, 40, sessions - 4)])
    c = Cache(rng, lens, 2, 64, [([0, 1], 3), ([2, 3], 2)], layers=2)
    starts, members, prefix = [0, 2, 4], [0, 1, 2, 3], [3, 2]
    if what == "twice":
        members[3] = 1
    elif what == "outside":
        members[0] = sessions
    elif what == "negative":
        members[2] = -1
    elif what == "falling":
        starts[1] = 5
    elif what == "open start":
        starts[0] = 1
    elif what == "open end":
        starts[2] = 3
    elif what == "long prefix":
        prefix[1] = c.tables.shape[1] + 1
    else:
        prefix[0] = -1
    pool = c.device(kv)
    q = W.normal_bf16(rng, (sessions, 8, 64))
    w0, p0 = c.entries(rng)
    weights, positions = torch.from_numpy(w0).cuda(), torch.from_numpy(p0).cuda()
    ws = torch.full((kv.decode_weights_workspace_bytes(pool, sessions, 8, 2, 4),), 255, dtype=torch.uint8, device="cuda")
    out = torch.full((sessions, 8, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    arrays = i32_dev(starts), i32_dev(members), i32_dev(prefix)
    lens, reused = i32_dev(c.lens), i32_dev(np.maximum(c.lens - 1, 0))

    def call(groups):
        kv.paged_attn_decode_weights(pool, 1, bf16_dev(q), c.dtables, lens, 0.125, out, weights, positions, ws, reused_lens=reused,
                                     group_starts=groups[0], group_members=groups[1], prefix_blocks=groups[2])
    call(arrays)
    assert kv.ls_device_errors() == kv.LS_DEVERR_GROUP
    assert_within(out, *decode_reference(c, 1, q, 0.125)[:3], 64, what)
    assert np.array_equal(weights.cpu().numpy(), w0) and np.array_equal(positions.cpu().numpy(), p0)
    # the same workspace afterwards, with groups that can be: own keys get their weights
    call(c.group_arrays())
    assert kv.ls_device_errors() == 0
    changed = (weights.cpu().numpy() != w0)[1]
    for s, n in enumerate(c.lens):
        t = np.arange(n)
        got = changed[c.tables[s, t // BLOCK], :, t % BLOCK].any(1)
        assert not got[:c.prefix_of(s)].any() and got[max(n - 1, c.prefix_of(s)):].all()
