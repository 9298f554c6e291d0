"""The binding's calls of the 8-bit cache launch on the current device: with any one of their tensors on another one, nothing is launched.  (Stand-ins for
tensors; the library is one that counts its calls.)"""
import types

import pytest
import torch

from paper_2602_23200_amd import binding as iq

B, HQ, HK, T, D = 2, 4, 2, 3, 128


class Stand:
    is_cuda = True

    def __init__(self, *shape, dtype=torch.float16):
        self.shape, self.dtype, self.place = torch.Size(shape), dtype, 0
        self.strides = torch.empty(shape, dtype=dtype, device="meta").stride()
        self.nbytes = 1 << 30

    def stride(self):
        return self.strides

    def data_ptr(self):
        return 4096

    def get_device(self):
        return self.place

    def is_contiguous(self):
        return True

    def element_size(self):
        return self.dtype.itemsize


@pytest.fixture
def calls(monkeypatch):
    made = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: made.append(name) or iq.OK

    monkeypatch.setattr(iq, "lib", lambda: Library())
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 0, raising=False)
    return made


def all_calls():
    """Name, tensors by name, the call."""
    cfg = iq.make_block_config(B, HQ, HK, capacity_tokens=64)
    new = lambda: dict(k=Stand(B, HK, T, D), v=Stand(B, HK, T, D))  # noqa: E731
    counts = lambda: dict(n=Stand(B, dtype=torch.int32), t=Stand(B, dtype=torch.int32))  # noqa: E731
    result = lambda: dict(q=Stand(B, HQ, T, D), ws=Stand(1, dtype=torch.uint8), out=Stand(B, HQ, T, D))  # noqa: E731
    cache = types.SimpleNamespace(cfg=cfg, buffers={"k_codes": Stand(1, dtype=torch.uint8)}, c=iq.innerq_block_cache_t())
    return cache, [
        ("append", new(), lambda a: iq.innerq_block_append(cache, a["k"], a["v"])),
        ("append_ragged", {**new(), **counts()}, lambda a: iq.innerq_block_append_ragged(cache, a["n"], a["t"], a["k"], a["v"])),
        ("read", new(), lambda a: iq.innerq_block_read(cache, 0, a["k"], a["v"])),
        ("read_ragged", {**new(), **counts()}, lambda a: iq.innerq_block_read_ragged(cache, a["n"], a["t"], a["k"], a["v"])),
        ("attention", {**new(), **result()}, lambda a: iq.innerq_block_attention(cache, a["k"], a["v"], a["q"], a["ws"], out=a["out"])),
        ("attention_ragged", {**new(), **result(), **counts()},
         lambda a: iq.innerq_block_attention_ragged(cache, a["n"], a["t"], 64, a["k"], a["v"], a["q"], a["ws"], out=a["out"])),
        ("cross_attention", result(), lambda a: iq.innerq_block_cross_attention(cache, a["q"], a["ws"], out=a["out"])),
        ("cross_attention_ragged", {**result(), **counts()},
         lambda a: iq.innerq_block_cross_attention_ragged(cache, a["n"], a["t"], 64, a["q"], a["ws"], out=a["out"]))]


@pytest.mark.parametrize("which", range(8))
def test_any_tensor_of_another_device_is_refused(calls, which):
    cache, every = all_calls()
    name, tensors, call = every[which]
    call(tensors)
    assert calls == ["innerq_block_" + name]
    for what, t in [*tensors.items(), ("the cache", cache.buffers["k_codes"])]:
        t.place = 1
        with pytest.raises(AssertionError):
            call(tensors)
        t.place = 0
    assert len(calls) == 1
    call(tensors)
    assert len(calls) == 2


def test_a_page_table_of_another_device_is_refused():
    cfg = iq.make_block_config(1, 2, 2, capacity_tokens=64, page_pool_pages=1)
    table = torch.zeros(1, 1, dtype=torch.int32)
    with pytest.raises(AssertionError):
        iq.allocate_block_cache(cfg, device="meta", page_table=table)
    assert iq.allocate_block_cache(cfg, device="cpu", page_table=table).n_tokens == 0
