"""Paged cache entry points, host side: what they refuse before anything is launched, and their workspace queries."""
import ctypes

import pytest

from paper_2603_30033_b200 import binding as Bd
from paper_2603_30033_b200 import build as Bu

FAKE = ctypes.c_void_p(4096)          # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    Bu.build()
    return Bd.load_library()


def desc(**kw):
    base = dict(B=2, N=1, d_model=128, n_H=4, r=(2, 16, 16), t=(2, 16, 16), causal=True, rope=True, dtype=Bd.TA_DTYPE_F32)
    base.update(kw)
    return Bd.make_desc(**base)


def cache(K=4096, V=8192, table=4096, n_pages=8, page_size=16, max_pages=4):
    return Bd.TuckerPagedCache(K, V, table, n_pages, page_size, max_pages)


def decode(lib, d=None, c=None, x=FAKE, w=FAKE, ut3=None, lens=FAKE, ptab=FAKE, plen=20, y=FAKE, ws=FAKE, n=1 << 30):
    d, c = d or desc(), c or cache()
    ut3 = ut3 or ctypes.c_void_p(12288)
    return lib.tucker_attn_decode_prefix(ctypes.byref(d), x, w, w, w, w, w, w, w, ut3, ctypes.byref(c), lens, ptab, plen, 1, y, ws, n, None)


def append(lib, d=None, c=None, X=FAKE, U3=FAKE, Ut3=None, lens=FAKE, start=FAKE, T=5, ws=FAKE, n=1 << 30):
    d, c = d or desc(), c or cache()
    return lib.tucker_cache_append_paged(ctypes.byref(d), X, U3, Ut3 or ctypes.c_void_p(12288), ctypes.byref(c), lens, start, T, ws, n, None)


BAD_CACHES = [dict(K=None), dict(V=None), dict(table=None), dict(n_pages=0), dict(page_size=0), dict(max_pages=0), dict(page_size=-16),
              dict(K=4100), dict(V=8200), dict(max_pages=1 << 20, page_size=1 << 12), dict(V=4096)]


@pytest.mark.parametrize("bad", BAD_CACHES, ids=str)
def test_bad_caches(lib, bad):
    assert decode(lib, c=cache(**bad)) == -1
    assert append(lib, c=cache(**bad)) == -1


def test_bad_decode_arguments(lib):
    for kw in (dict(x=None), dict(w=None), dict(lens=None), dict(ptab=None), dict(plen=-1), dict(y=None), dict(ws=None),
               dict(x=ctypes.c_void_p(4098)), dict(ws=ctypes.c_void_p(4096 + 16)), dict(d=desc(B=0)), dict(d=desc(r=(2, 16, 15))),
               dict(d=desc(n_H=3)), dict(plen=(1 << 31) - 1)):
        assert decode(lib, **kw) == -1, kw
    assert decode(lib, n=16) == -3
    assert decode(lib, d=desc(t=(2, 16, 4096))) == -2                     # a value rank no kernel covers
    assert decode(lib, d=desc(B=70000)) == -2
    assert lib.tucker_attn_decode_prefix(None, *[FAKE] * 9, ctypes.byref(cache()), FAKE, None, 0, 1, FAKE, FAKE, 1, None) == -1
    assert lib.tucker_attn_decode_paged(ctypes.byref(desc()), *[FAKE] * 9, None, FAKE, 1, FAKE, FAKE, 1 << 30, None) == -1


def test_bad_append_arguments(lib):
    for kw in (dict(X=None), dict(U3=None), dict(lens=None), dict(start=None), dict(T=-1), dict(ws=None), dict(ws=ctypes.c_void_p(4112)), dict(X=ctypes.c_void_p(4104)),
               dict(d=desc(pos0=-1)), dict(d=desc(pos0=(1 << 31) - 1)), dict(d=desc(r=(2, 16, 15)))):
        assert append(lib, **kw) == -1, kw


    assert append(lib, n=16) == -3


def test_workspace_queries(lib):
    tokens = lambda d, T: lib.tucker_cache_append_paged_workspace_bytes(ctypes.byref(d), ctypes.byref(cache()), T)
    assert tokens(desc(), 0) > 0 and tokens(desc(), 5) > 0 and tokens(desc(), -1) == 0 and tokens(desc(B=0), 5) == 0
    big = desc(d_model=4096, n_H=32, r=(2, 128, 128), t=(2, 128, 128), dtype=Bd.TA_DTYPE_BF16)
    assert tokens(big, 1000) > 1000 * 256 * 4                              # partial sums of the shares of d
    need = lambda d, c, p: lib.tucker_attn_decode_prefix_workspace_bytes(ctypes.byref(d), ctypes.byref(c), p)
    paged = lambda d, c: lib.tucker_attn_decode_paged_workspace_bytes(ctypes.byref(d), ctypes.byref(c))
    assert paged(desc(), cache()) == need(desc(), cache(), 0) > 0
    assert need(desc(), cache(), 1000) > need(desc(), cache(), 0)
    assert need(desc(B=8), cache(), 100) > need(desc(), cache(), 100)
    assert need(desc(), cache(), -1) == 0 and need(desc(), cache(page_size=0), 0) == 0 and need(desc(B=-1), cache(), 0) == 0
    assert need(desc(t=(2, 16, 4096)), cache(), 0) == 0


def test_struct_layout():
    # three pointers, three 32-bit fields, tail padding
    assert ctypes.sizeof(Bd.TuckerPagedCache) == 40
