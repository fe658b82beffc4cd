"""The binding refuses cache operators whose parts are on several devices, or not on the current one, before
anything of the library is called. Stand-ins for tensors' owners: no GPU needed."""

import types

import pytest
import torch


def parts(cache=0, batch=0, workspace=0):
    def on(index, **more):
        device = torch.device("cuda", index)
        return types.SimpleNamespace(device=device, index=index, tensor=types.SimpleNamespace(device=device), **more)

    return (on(cache, heads=2, dim=128, ref=None, struct=None), on(batch, tokens=1, ref=None, struct=None),
            on(workspace, address=256, bytes=1 << 20))


@pytest.fixture
def binding(fsb, monkeypatch):
    """The binding with a library that must not be reached, device 0 current."""

    def reached():
        raise AssertionError("the library was called")

    monkeypatch.setattr(fsb, "lib", reached)
    monkeypatch.setattr(fsb, "_current_device", lambda: 0, raising=False)
    monkeypatch.setattr(fsb, "_current_stream", lambda index: 0)

    class Row:  # (what the binding asks of a tensor; on the cache's device, so that only the devices are wrong)
        dtype, shape = torch.bfloat16, (1, 2, 128)

        def __init__(self, index):
            self.index = index

        def stride(self):
            return (256, 128, 1)

        def get_device(self):
            return self.index

        def data_ptr(self):
            return 4096

        def numel(self):
            return 256

    return fsb, Row


OTHERS = [(dict(batch=1), "batch is on cuda:1"), (dict(workspace=1), "workspace is on cuda:1"),
          (dict(cache=1, batch=1, workspace=1), "cuda:0 is current")]


@pytest.mark.parametrize("where,word", OTHERS)
def test_append_and_attend(binding, where, word):
    fsb, Row = binding
    c, b, w = parts(**where)
    x = Row(c.device.index)
    with pytest.raises(ValueError, match=word):
        fsb.fs_kv_append(c, b, x, x, workspace=w)
    with pytest.raises(ValueError, match=word):
        fsb.fs_kv_attend(c, b, x, x, 0.1, workspace=w)


def test_workspace_and_check(binding):
    fsb, _ = binding
    c, b, w = parts(batch=1)
    with pytest.raises(ValueError, match="batch is on cuda:1"):
        fsb.KvWorkspace(c, b, 2)
    c, b, w = parts(1, 1, 1)
    with pytest.raises(ValueError, match="cuda:0 is current"):
        fsb.KvWorkspace(c, b, 2)
    with pytest.raises(ValueError, match="cuda:0 is current"):
        fsb.fs_kv_check(w)


def test_one_device_goes_on_to_the_library(binding):
    fsb, Row = binding
    c, b, w = parts()
    x = Row(0)
    for call in (lambda: fsb.fs_kv_append(c, b, x, x, workspace=w), lambda: fsb.fs_kv_attend(c, b, x, x, 0.1, workspace=w),
                 lambda: fsb.fs_kv_check(w)):
        with pytest.raises(AssertionError, match="the library was called"):
            call()
