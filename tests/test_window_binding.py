"""The binding's checks of tensors in the windowed calls: each refusal is a ValueError, before the library is called."""
import pytest
import torch


class Tensor:
    """What the checks read of a device tensor, without a device."""

    def __init__(self, *shape, dtype=torch.int32, device=0):
        self.shape, self.dtype, self.device_index = torch.Size(shape), dtype, device
        self.is_cuda = device >= 0

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return True

    def get_device(self):
        return self.device_index

    def element_size(self):
        return self.dtype.itemsize

    def stride(self, i=None):
        s = [1]
        for n in reversed(self.shape[1:]):
            s.insert(0, s[0] * n)
        return tuple(s[:self.dim()]) if i is None else s[i]

    def data_ptr(self):
        return 0x10000


def i64(*shape, **kw):
    return Tensor(*shape, dtype=torch.int64, **kw)


def bf16(*shape, **kw):
    return Tensor(*shape, dtype=torch.bfloat16, **kw)


@pytest.fixture
def kv(built_lib, monkeypatch):
    from paper_2606_22983_amd import kv as kv_mod

    class Called(Exception):
        pass

    class Library:
        def __getattr__(self, name):
            def call(*args):
                raise Called(name)
            return call
    monkeypatch.setattr(kv_mod, "_lib", Library())
    monkeypatch.setattr(kv_mod, "_stream", lambda stream: None)
    kv_mod.Called = Called
    yield kv_mod
    del kv_mod.Called


@pytest.fixture
def pool(kv):
    p = kv.KVPool(None, bf16(4096), 1, 4, 2, 64, 16)
    return p


def calls(kv, pool):
    """Each entry point with its tensors, by name."""
    s = 3
    tables = dict(seq_lens=Tensor(s), new_lens=Tensor(s), block_tables=Tensor(s, 4), next_lens=Tensor(s), cu_new_lens=Tensor(s + 1),
                  reused_lens=Tensor(s), slot_map=i64(5), free_ring=Tensor(8), free_counts=i64(2), next_counts=i64(2))
    append = dict(k_new=bf16(5, 2, 64), v_new=bf16(5, 2, 64), slot_map=i64(5))
    rows = dict(q=bf16(s, 4, 64), block_tables=Tensor(s, 4), out=bf16(s, 4, 64), k_new=bf16(s, 2, 64), v_new=bf16(s, 2, 64),
                workspace=Tensor(4096, dtype=torch.uint8))
    decode = dict(rows, context_lens=Tensor(s))
    prefill = dict(rows, cu_new_lens=Tensor(s + 1), reused_lens=Tensor(s))
    return [(lambda **t: kv.kv_tables_update(pool, max_new_len=2, window=16, **t), tables),
            (lambda **t: kv.kv_append(pool, 0, **t), append),
            (lambda **t: kv.paged_attn_decode_window(pool, 0, window=16, sinks=0, scale=0.125, **t), decode),
            (lambda **t: kv.paged_attn_prefill_window(pool, 0, max_new_len=2, window=16, sinks=0, scale=0.125, **t), prefill)]


def test_good_tensors_reach_the_library(kv, pool):
    for call, tensors in calls(kv, pool):
        with pytest.raises(kv.Called):
            call(**tensors)


def test_tensors_without_dimensions(kv, pool):
    for call, tensors in calls(kv, pool):
        for name, t in tensors.items():
            if name != "workspace":                   # (any shape)
                with pytest.raises(ValueError):
                    call(**dict(tensors, **{name: Tensor(dtype=t.dtype)}))


def test_tensors_of_another_shape_or_type(kv, pool):
    for call, tensors in calls(kv, pool):
        for name, t in tensors.items():
            if name == "workspace":
                continue
            others = [Tensor(*t.shape, 1, dtype=t.dtype), Tensor(*t.shape, dtype=torch.float32)]
            if name not in ("free_ring", "slot_map"):  # (any length)
                others.append(Tensor(t.shape[0] + 1, *t.shape[1:], dtype=t.dtype))
            for other in others:
                with pytest.raises(ValueError):
                    call(**dict(tensors, **{name: other}))


def test_tensors_on_the_host(kv, pool):
    for call, tensors in calls(kv, pool):
        for name, t in tensors.items():
            with pytest.raises(ValueError):
                call(**dict(tensors, **{name: Tensor(*t.shape, dtype=t.dtype, device=-1)}))


def test_tensors_on_another_gpu(kv, pool):
    """Their memory is not the pool's device's: a kernel that reads it faults."""
    for call, tensors in calls(kv, pool):
        for name, t in tensors.items():
            with pytest.raises(ValueError, match="pool's device"):
                call(**dict(tensors, **{name: Tensor(*t.shape, dtype=t.dtype, device=1)}))
