"""Binding of the 8-bit calls without a GPU: tensors and library are stand-ins that record what happens in which order."""
import types

import pytest
import torch

from paper_2603_30033_b200 import binding as Bd
from tests.test_paged_binding_cpu import CALLS, Stand

NAMES = ("tucker_cache_append_paged_q8", "tucker_cache_store_paged_q8", "tucker_cache_read_paged_q8", "tucker_attn_decode_prefix_q8")


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

    lib = types.SimpleNamespace(**{n: note("call", 0) for n in NAMES},
                                **{n + "_workspace_bytes": note("query", 1 << 20) for n in (NAMES[0], NAMES[3])})
    monkeypatch.setattr(Bd, "load_library", lambda: lib)
    monkeypatch.setattr(Bd, "_enter_device", enter)
    monkeypatch.setattr(Bd, "_stream_ptr", lambda device: 0)
    monkeypatch.setattr(Bd, "alloc_workspace", lambda n, device: (log.append(("alloc", current[0])), Stand(n, dtype=torch.uint8))[1])
    return log


def i32(*s):
    return Stand(*s, dtype=torch.int32)


def cache(r, t):
    c = lambda n: Stand(4, 16, n, dtype=torch.float8_e4m3fn)
    s = lambda: Stand(4, 16, dtype=torch.float8_e8m0fnu)
    return c(r), s(), c(t), s()


def weights(r=64):
    return [Stand(2, 32, r), Stand(4, 2), Stand(64, 32), Stand(64, r), Stand(2, 32, r), Stand(4, 2), Stand(64, 32), Stand(64, r)]


def test_append_on_the_device_of_the_call(recorded):
    Bd.tucker_cache_append_paged_q8(Stand(5, 64), Stand(64, 32), Stand(64, 32), *cache(32, 32), i32(2, 3), i32(2), i32(3), rope=True)
    assert recorded == CALLS


@pytest.mark.parametrize("read", [False, True])
def test_rows_on_the_device_of_the_call(recorded, read):
    K, Ks, V, Vs = cache(32, 48)
    k, v = Stand(5, 32), Stand(5, 48)
    if read:
        Bd.tucker_cache_read_paged_q8(K, Ks, V, Vs, i32(2, 3), i32(2), i32(3), k, v)
    else:
        Bd.tucker_cache_store_paged_q8(k, v, K, Ks, V, Vs, i32(2, 3), i32(2), i32(3))
    assert recorded == [("call", 1), ("leave", 0)]


@pytest.mark.parametrize("prefix", [False, True])
def test_decode_on_the_device_of_the_call(recorded, prefix):
    args = (Stand(2, 64), *weights(), *cache(64, 64), i32(2, 3), i32(2))
    if prefix:
        Bd.tucker_attn_decode_prefix_q8(*args, i32(2), 20, n_H=4, rope=True, out=Stand(2, 64))
    else:
        Bd.tucker_attn_decode_paged_q8(*args, n_H=4, rope=True, out=Stand(2, 64))
    assert recorded == CALLS


def test_an_own_workspace_is_not_asked_for(recorded):
    Bd.tucker_attn_decode_paged_q8(Stand(2, 64), *weights(), *cache(64, 64), i32(2, 3), i32(2), n_H=4, rope=True, out=Stand(2, 64),
                                   workspace=Stand(1 << 20, dtype=torch.uint8))
    assert recorded == [("call", 1), ("leave", 0)]


@pytest.mark.parametrize("bad", ["codes", "scales", "rows of scales", "another device", "table", "short prefix table"])
def test_refusals(recorded, bad):
    K, Ks, V, Vs = cache(64, 64)
    table, ptab = i32(2, 3), i32(2)
    if bad == "codes":
        K.dtype = torch.uint8
    if bad == "scales":
        Vs.dtype = torch.uint8
    if bad == "rows of scales":
        Ks.shape = torch.Size((4, 15))
    if bad == "another device":
        V.device, V.get_device = torch.device("cuda", 0), lambda: 0
    if bad == "table":
        table = i32(3, 3)
    if bad == "short prefix table":
        ptab = i32(1)
    with pytest.raises((ValueError, TypeError)):
        Bd.tucker_attn_decode_prefix_q8(Stand(2, 64), *weights(), K, Ks, V, Vs, table, i32(2), ptab, 20, n_H=4, rope=True, out=Stand(2, 64))
    assert recorded == []
