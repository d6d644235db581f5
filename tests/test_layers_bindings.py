"""How the bindings call the library with a workspace, on stand-ins (no GPU): the device made current, the workspace taken on the
call's stream and given back whatever the call says, and none taken where none is needed."""
import contextlib
import types

import pytest
import torch

from paper_2010_11305_amd import dense_lib as lib
from paper_2010_11305_amd import emb_cache


@pytest.fixture
def seen(monkeypatch):
    log, state = [], {"device": 0, "status": 0}

    @contextlib.contextmanager
    def device(index):
        was, state["device"] = state["device"], index
        log.append(("device", index))
        yield
        state["device"] = was

    def f(*args):
        log.append(("call", state["device"], *args))
        return state["status"]

    monkeypatch.setattr(lib, "_lib", types.SimpleNamespace(f=f))
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: state["device"], raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 1000 + index, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_cudaCachingAllocator_raw_alloc",
                        lambda n, stream: log.append(("alloc", state["device"], n, stream)) or 4096, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_cudaCachingAllocator_raw_delete", lambda p: log.append(("delete", p)), raising=False)
    return log, state


def test_on_the_current_device(seen):
    log, _ = seen
    lib.call_in("f", torch.device("cuda", 0), 512, 7, 8)
    assert log == [("alloc", 0, 512, 1000), ("call", 0, 7, 8, 4096, 512, 1000), ("delete", 4096)]


def test_on_another_device(seen):
    log, state = seen
    lib.call_in("f", torch.device("cuda", 3), 512, 7)
    assert log == [("device", 3), ("alloc", 3, 512, 1003), ("call", 3, 7, 4096, 512, 1003), ("delete", 4096)] and state["device"] == 0
    log.clear()
    lib.call_in("f", torch.device("cuda", 3), 0, 7)
    assert log == [("device", 3), ("call", 3, 7, None, 0, 1003)]


def test_without_a_workspace(seen):
    log, _ = seen
    lib.call_in("f", torch.device("cuda", 0), 0, 7)
    assert log == [("call", 0, 7, None, 0, 1000)]


def test_a_refused_call_gives_it_back(seen):
    log, state = seen
    state["status"] = emb_cache.EMB_EINVAL
    with pytest.raises(emb_cache.EmbCacheError):
        lib.call_in("f", torch.device("cuda", 0), 256)
    assert log[-1] == ("delete", 4096)
