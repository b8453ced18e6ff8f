"""The binding's checks of tensors for shared prefixes, accumulated weights and eviction: each refusal is a ValueError,
before the library is called."""
import pytest
import torch

from tests.test_window_binding import Tensor, bf16, i64, kv  # noqa: F401  (fixture)


def f32(*shape, **kw):
    return Tensor(*shape, dtype=torch.float32, **kw)


class Pool:
    handle, device, num_layers, num_blocks, num_kv_heads, head_dim, block_size = 1, 0, 2, 10, 2, 64, 16


ENTRY = (2, 10, 2, 16)


def shared(kv, **kw):  # noqa: F811
    a = dict(q=bf16(4, 8, 64), bt=Tensor(4, 6), lens=Tensor(4), starts=Tensor(3), members=Tensor(4), prefix=Tensor(2),
             out=bf16(4, 8, 64), ws=Tensor(1000))
    a.update(kw)
    kv.paged_attn_decode_shared(Pool, 0, a["q"], a["bt"], a["lens"], a["starts"], a["members"], a["prefix"], 0.1, a["out"], a["ws"])


def weights(kv, **kw):  # noqa: F811
    a = dict(q=bf16(4, 8, 64), bt=Tensor(4, 6), lens=Tensor(4), out=bf16(4, 8, 64), w=f32(*ENTRY), pos=Tensor(*ENTRY), ws=Tensor(1000),
             reused=Tensor(4), begin=Tensor(4), first=Tensor(4), starts=Tensor(3), members=Tensor(4), prefix=Tensor(2))
    a.update(kw)
    kv.paged_attn_decode_weights(Pool, 0, a["q"], a["bt"], a["lens"], 0.1, a["out"], a["w"], a["pos"], a["ws"], a["reused"], a["begin"],
                                 a["first"], a["starts"], a["members"], a["prefix"])


def prompt(kv, **kw):  # noqa: F811
    a = dict(q=bf16(9, 8, 64), cu=Tensor(5), ctx=Tensor(4), bt=Tensor(4, 6), w=f32(*ENTRY), pos=Tensor(*ENTRY), ws=Tensor(1000),
             begin=Tensor(4), first=Tensor(4))
    a.update(kw)
    kv.kv_weights_prefill(Pool, 0, a["q"], a["cu"], a["ctx"], 5, a["bt"], 3, 0.1, a["w"], a["pos"], a["ws"], a["begin"], a["first"])


def evict(kv, **kw):  # noqa: F811
    a = dict(lens=Tensor(4), bt=Tensor(4, 6), nextp=Tensor(4), w=f32(*ENTRY), pos=Tensor(*ENTRY), nextl=Tensor(4), wn=f32(*ENTRY),
             pn=Tensor(*ENTRY), first=Tensor(4), ring=Tensor(20), counts=i64(2), after=i64(2))
    a.update(kw)
    kv.kv_evict(Pool, a["lens"], a["bt"], 10, 12, 3, a["nextp"], a["w"], a["pos"], a["nextl"], a["wn"], a["pn"], a["first"],
                free_ring=a["ring"], free_counts=a["counts"], next_counts=a["after"])


GROUPS = [dict(starts=None), dict(members=None), dict(prefix=None), dict(starts=Tensor(2)), dict(starts=Tensor(1, 3)),
          dict(prefix=Tensor(2, 1)), dict(prefix=Tensor()), dict(members=Tensor(2, 2)), dict(members=i64(4)), dict(prefix=i64(2)),
          dict(starts=Tensor(3, device=1)), dict(members=Tensor(4, device=-1))]
ENTRIES = [dict(w=f32(2, 10, 2, 8)), dict(w=f32(1, 10, 2, 16)), dict(w=bf16(*ENTRY)), dict(w=f32(*ENTRY, device=1)),
           dict(pos=i64(*ENTRY)), dict(pos=Tensor(2, 10, 32)), dict(pos=Tensor(*ENTRY, device=-1))]
ROWS = [dict(q=bf16(4, 8)), dict(q=bf16(4, 8, 128)), dict(q=f32(4, 8, 64)), dict(q=bf16(4, 8, 64, device=1)), dict(bt=Tensor(3, 6)),
        dict(bt=Tensor(24)), dict(lens=Tensor(5)), dict(lens=i64(4)), dict(lens=Tensor(4, device=1)), dict(out=bf16(4, 7, 64)),
        dict(out=bf16(4, 8, 64, device=-1)), dict(ws=Tensor(10, device=1)), dict(ws=Tensor(10, device=-1))]


@pytest.mark.parametrize("kw", ROWS + GROUPS)
def test_decode_shared(kv, kw):  # noqa: F811
    with pytest.raises(ValueError):
        shared(kv, **kw)


@pytest.mark.parametrize("kw", ROWS + GROUPS + ENTRIES + [
    dict(reused=Tensor(3)), dict(reused=i64(4)), dict(begin=Tensor(4, 1)), dict(begin=Tensor(4, device=1)), dict(first=Tensor(5)),
    dict(first=Tensor())])
def test_decode_weights(kv, kw):  # noqa: F811
    with pytest.raises(ValueError):
        weights(kv, **kw)


@pytest.mark.parametrize("kw", ENTRIES + [
    dict(q=bf16(9, 64)), dict(q=bf16(9, 8, 32)), dict(q=f32(9, 8, 64)), dict(cu=Tensor(4)), dict(cu=i64(5)), dict(ctx=Tensor(4, 1)),
    dict(ctx=Tensor(3)), dict(ctx=Tensor()), dict(bt=Tensor(4)), dict(bt=Tensor(5, 6)), dict(begin=Tensor(3)), dict(first=i64(4)),
    dict(ws=Tensor(10, device=1)), dict(q=bf16(9, 8, 64, device=-1))])
def test_weights_prefill(kv, kw):  # noqa: F811
    with pytest.raises(ValueError):
        prompt(kv, **kw)


@pytest.mark.parametrize("kw", ENTRIES + [
    dict(lens=Tensor(4, 1)), dict(lens=Tensor()), dict(lens=i64(4)), dict(bt=Tensor(3, 6)), dict(bt=Tensor(6)), dict(nextp=Tensor(3)),
    dict(nextl=Tensor(5)), dict(nextl=i64(4)), dict(wn=f32(2, 10, 2, 4)), dict(wn=Tensor(*ENTRY)), dict(pn=f32(*ENTRY)),
    dict(pn=Tensor(*ENTRY, device=1)), dict(first=Tensor(2)), dict(ring=Tensor(4, 5)), dict(ring=i64(20)), dict(counts=Tensor(2)),
    dict(counts=i64(3)), dict(after=i64(2, device=1))])
def test_evict(kv, kw):  # noqa: F811
    with pytest.raises(ValueError):
        evict(kv, **kw)


def test_what_may_be_left_out_reaches_the_library(kv):  # noqa: F811
    none = dict(starts=None, members=None, prefix=None)
    for call, kw in ((shared, {}), (shared, none), (weights, {}), (weights, dict(none, reused=None, begin=None, first=None, pos=None)),
                     (prompt, {}), (prompt, dict(begin=None, first=None)), (evict, {}),
                     (evict, dict(wn=None, pn=None, first=None, ring=None, counts=None, after=None))):
        with pytest.raises(kv.Called):
            call(kv, **kw)
