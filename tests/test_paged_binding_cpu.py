"""Binding of the paged calls without a GPU: tensors and library are stand-ins that record what happens in which order."""
import types

import pytest
import torch

from paper_2603_30033_b200 import binding as Bd


class Stand:
    """What the binding asks of a contiguous CUDA tensor on device 1."""
    is_cuda = True
    device = torch.device("cuda", 1)

    def __init__(self, *shape, dtype=torch.bfloat16):
        self.shape, self.dtype = torch.Size(shape), dtype

    def dim(self):
        return len(self.shape)

    def get_device(self):
        return 1

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096

    def numel(self):
        return self.shape.numel()


@pytest.fixture
def recorded(monkeypatch):
    """The list of (what, current device) that a call leaves, with device 0 current in front of it."""
    log, current = [], [0]

    class Guard:
        def __exit__(self, *_):
            current[0] = 0
            log.append(("leave", current[0]))

    def enter(cuda, device):
        current[0] = device.index
        return Guard()

    def note(what, result):
        def f(*_):
            log.append((what, current[0]))
            return result
        return f

    lib = types.SimpleNamespace(tucker_cache_append_paged_workspace_bytes=note("query", 1 << 20), tucker_cache_append_paged=note("call", 0),
                                tucker_attn_decode_prefix_workspace_bytes=note("query", 1 << 20), tucker_attn_decode_prefix=note("call", 0))
    monkeypatch.setattr(Bd, "load_library", lambda: lib)
    monkeypatch.setattr(Bd, "_enter_device", enter)
    monkeypatch.setattr(Bd, "_stream_ptr", lambda device: 0)
    monkeypatch.setattr(Bd, "alloc_workspace", lambda n, device: (log.append(("alloc", current[0])), Stand(n, dtype=torch.uint8))[1])
    return log


CALLS = [("query", 1), ("alloc", 1), ("call", 1), ("leave", 0)]


def test_append_asks_for_its_workspace_on_the_device_of_the_call(recorded):
    i = lambda *s: Stand(*s, dtype=torch.int32)
    Bd.tucker_cache_append_paged(Stand(5, 64), Stand(64, 32), Stand(64, 32), Stand(4, 16, 32), Stand(4, 16, 32), i(2, 3), i(2), i(3), rope=True)
    assert recorded == CALLS


def test_decode_asks_for_its_workspace_on_the_device_of_the_call(recorded):
    i = lambda *s: Stand(*s, dtype=torch.int32)
    weights = [Stand(2, 32, 64), Stand(4, 2), Stand(64, 32), Stand(64, 64), Stand(2, 32, 64), Stand(4, 2), Stand(64, 32), Stand(64, 64)]
    Bd.tucker_attn_decode_paged(Stand(2, 64), *weights, Stand(4, 16, 64), Stand(4, 16, 64), i(2, 3), i(2), n_H=4, rope=True, out=Stand(2, 64))
    assert recorded == CALLS
