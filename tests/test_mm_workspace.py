"""A workspace is ready for calls on any stream when its constructor returns (stand-ins for CUDA: no GPU needed)."""

import ctypes as C
import types

import pytest
import torch


class Device:
    """torch's CUDA calls as a constructor makes them: memory comes full of 7, a wait notes what memory holds by then."""

    def __init__(self, monkeypatch, fsb, capturing):
        self.memory, self.seen = None, []
        monkeypatch.setattr(torch, "empty", self.empty)
        monkeypatch.setattr(torch, "zeros", lambda n, **more: self.empty(n, **more).zero_())
        monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda *device: self)
        monkeypatch.setattr(fsb, "_current_device", lambda: 0, raising=False)

    def empty(self, n, dtype, device):
        self.memory = torch.full((n,), 7, dtype=dtype)
        return self.memory

    def synchronize(self):
        self.seen.append(self.memory.clone())


@pytest.mark.parametrize("backward", [False, True])
def test_products(fsb, monkeypatch, backward):
    d = Device(monkeypatch, fsb, False)
    work = fsb.MmWorkspace(300, 200, 500, backward=backward)
    n = C.c_int64()
    fsb.lib().fs_mm_workspace_bytes(300, 200, 500, backward, C.byref(n))
    assert len(d.memory) == work.bytes == n.value
    assert len(d.seen) == 1 and not d.seen[0][:256].any()  # what has to be zero is, before anyone can call
    assert bool((d.memory[256:] == 7).all())  # the rest is written by calls alone


def test_products_within_a_capture(fsb, monkeypatch):
    """A stream that is being captured cannot be waited for: the fill is captured with what follows it."""
    d = Device(monkeypatch, fsb, True)
    fsb.MmWorkspace(300, 200, 500, backward=True)
    assert not d.seen and not d.memory[:256].any()


def test_the_cache_operators(fsb, monkeypatch):
    d = Device(monkeypatch, fsb, False)

    def workspace_bytes(cache, batch, q_heads, n):  # (the library's asks for a device)
        n._obj.value = 70000
        return fsb.FS_OK

    monkeypatch.setattr(fsb, "lib", lambda: types.SimpleNamespace(fs_kv_workspace_bytes=workspace_bytes))
    on = lambda struct: types.SimpleNamespace(struct=struct, index=0, device="cuda:0")  # noqa: E731
    work = fsb.KvWorkspace(on(fsb.fs_kv_cache()), on(fsb.fs_kv_batch()), 16)
    assert len(d.memory) == work.bytes == 70000
    assert len(d.seen) == 1 and not d.seen[0].any()
