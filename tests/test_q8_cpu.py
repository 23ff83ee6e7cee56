"""8-bit paged cache, host side: the format's arithmetic, what the entry points refuse before anything is launched, and their
workspace queries."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2603_30033_b200 import binding as Bd
from paper_2603_30033_b200 import build as Bu
from tests import q8_helpers as Q

FAKE = ctypes.c_void_p(4096)          # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    Bu.build()
    return Bd.load_library()


def desc(**kw):
    base = dict(B=2, N=1, d_model=128, n_H=4, r=(2, 16, 16), t=(2, 16, 16), causal=True, rope=True, dtype=Bd.TA_DTYPE_F32)
    base.update(kw)
    return Bd.make_desc(**base)


def cache(K=4096, V=8192, Ks=1 << 14, Vs=1 << 15, table=4096, n_pages=8, page_size=16, max_pages=4):
    return Bd.TuckerPagedCacheQ8(K, V, Ks, Vs, table, n_pages, page_size, max_pages)


def decode(lib, d=None, c=None, x=FAKE, w=FAKE, ut3=None, lens=FAKE, ptab=FAKE, plen=20, y=FAKE, ws=FAKE, n=1 << 30):
    d, c = d or desc(), c or cache()
    ut3 = ut3 or ctypes.c_void_p(12288)
    return lib.tucker_attn_decode_prefix_q8(ctypes.byref(d), x, w, w, w, w, w, w, w, ut3, ctypes.byref(c), lens, ptab, plen, 1, y, ws, n, None)


def append(lib, d=None, c=None, X=FAKE, U3=FAKE, Ut3=None, lens=FAKE, start=FAKE, T=5, ws=FAKE, n=1 << 30):
    d, c = d or desc(), c or cache()
    return lib.tucker_cache_append_paged_q8(ctypes.byref(d), X, U3, Ut3 or ctypes.c_void_p(12288), ctypes.byref(c), lens, start, T, ws, n, None)


def store(lib, d=None, c=None, K=FAKE, V=ctypes.c_void_p(8192), lens=FAKE, start=FAKE, T=5):
    d, c = d or desc(), c or cache()
    return lib.tucker_cache_store_paged_q8(ctypes.byref(d), K, V, ctypes.byref(c), lens, start, T, None)


def read(lib, d=None, c=None, K=FAKE, V=ctypes.c_void_p(8192), lens=FAKE, start=FAKE, T=5):
    d, c = d or desc(), c or cache()
    return lib.tucker_cache_read_paged_q8(ctypes.byref(d), ctypes.byref(c), lens, start, T, K, V, None)


BAD_CACHES = [dict(K=None), dict(V=None), dict(Ks=None), dict(Vs=None), dict(table=None), dict(n_pages=0), dict(page_size=0), dict(max_pages=0),
              dict(page_size=-16), dict(K=4100), dict(V=8200), dict(Ks=(1 << 14) + 8), dict(Vs=(1 << 15) + 1),
              dict(max_pages=1 << 20, page_size=1 << 12),
              dict(V=4096),                          # one pool, two sets of scales
              dict(Vs=1 << 14),                      # two pools, one set of scales
              dict(V=4096, Vs=1 << 14)]              # one pool, but not one projection / not the same rows


@pytest.mark.parametrize("bad", BAD_CACHES, ids=str)
def test_bad_caches(lib, bad):
    assert decode(lib, c=cache(**bad)) == -1
    assert append(lib, c=cache(**bad)) == -1
    assert store(lib, c=cache(**bad)) == -1
    assert read(lib, c=cache(**bad)) == -1


def test_bad_decode_arguments(lib):
    for kw in (dict(x=None), dict(w=None), dict(lens=None), dict(ptab=None), dict(plen=-1), dict(y=None), dict(ws=None),
               dict(x=ctypes.c_void_p(4098)), dict(ws=ctypes.c_void_p(4096 + 16)), dict(d=desc(B=0)), dict(d=desc(r=(2, 16, 15))),
               dict(d=desc(n_H=3)), dict(plen=(1 << 31) - 1)):
        assert decode(lib, **kw) == -1, kw
    assert decode(lib, n=16) == -3
    assert decode(lib, d=desc(t=(2, 16, 4096))) == -2                     # a value rank no kernel covers
    assert decode(lib, d=desc(B=70000)) == -2
    assert lib.tucker_attn_decode_prefix_q8(None, *[FAKE] * 9, ctypes.byref(cache()), FAKE, None, 0, 1, FAKE, FAKE, 1, None) == -1
    assert lib.tucker_attn_decode_paged_q8(ctypes.byref(desc()), *[FAKE] * 9, None, FAKE, 1, FAKE, FAKE, 1 << 30, None) == -1


def test_bad_append_arguments(lib):
    for kw in (dict(X=None), dict(U3=None), dict(lens=None), dict(start=None), dict(T=-1), dict(ws=None), dict(ws=ctypes.c_void_p(4112)), dict(X=ctypes.c_void_p(4104)),
               dict(d=desc(pos0=-1)), dict(d=desc(pos0=(1 << 31) - 1)), dict(d=desc(r=(2, 16, 15)))):
        assert append(lib, **kw) == -1, kw
    assert append(lib, n=16) == -3
    assert append(lib, d=desc(t=(2, 16, 4096))) == -2


def test_bad_row_arguments(lib):
    for call in (store, read):
        for kw in (dict(K=None), dict(V=None), dict(K=ctypes.c_void_p(4104)), dict(V=ctypes.c_void_p(8194)), dict(lens=None), dict(start=None),
                   dict(T=-1), dict(d=desc(dtype=7)), dict(d=desc(B=0)), dict(c=cache(V=4096, Vs=1 << 14), d=desc(t=(2, 16, 32)), V=FAKE)):
            assert call(lib, **kw) == -1, kw
        assert call(lib, d=desc(t=(2, 16, 4096))) == -2
    assert read(lib, V=FAKE) == -1                   # two pools into one buffer


def test_workspace_queries(lib):
    tokens = lambda d, T: lib.tucker_cache_append_paged_q8_workspace_bytes(ctypes.byref(d), ctypes.byref(cache()), T)
    assert tokens(desc(), 0) > 0 and tokens(desc(), 5) > 0 and tokens(desc(), -1) == 0 and tokens(desc(B=0), 5) == 0
    need = lambda d, c, p: lib.tucker_attn_decode_prefix_q8_workspace_bytes(ctypes.byref(d), ctypes.byref(c), p)
    paged = lambda d, c: lib.tucker_attn_decode_paged_q8_workspace_bytes(ctypes.byref(d), ctypes.byref(c))
    assert paged(desc(), cache()) == need(desc(), cache(), 0) > 0
    assert need(desc(), cache(), -1) == 0 and need(desc(), cache(page_size=0), 0) == 0 and need(desc(B=-1), cache(), 0) == 0
    assert need(desc(t=(2, 16, 4096)), cache(), 0) == 0
    big = desc(B=64, d_model=4096, n_H=32, r=(2, 128, 128), t=(2, 128, 128), dtype=Bd.TA_DTYPE_BF16)
    assert need(big, cache(max_pages=512), 100000) > need(big, cache(max_pages=512), 0) > 1


def test_struct_layout():
    # five pointers, three 32-bit fields, tail padding
    assert ctypes.sizeof(Bd.TuckerPagedCacheQ8) == 56


def test_scale_bytes(tmp_path):
    """The header's host-callable arithmetic against the definition: numbers around every border, the smallest and largest, and
    those that are none."""
    src = tmp_path / "t.cu"
    src.write_text('#include <cstdio>\n#include <cstring>\n#include "ta_q8.cuh"\n'
                   'int main() { unsigned u; while (scanf("%x", &u) == 1) { const int b = ta::q8::scale_byte(u);\n'
                   '  printf("%d %x %x\\n", b, ta::q8::inverse_bits(b), ta::q8::scale_bits(b)); } }\n')
    exe = tmp_path / "t"
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run([Bu._nvcc(), "-std=c++17", "--expt-relaxed-constexpr", "-I", os.path.join(root, "include"), "-I",
                    os.path.join(root, "paper_2603_30033_b200", "csrc"), str(src), "-o", str(exe)], check=True, capture_output=True)
    rng = np.random.default_rng(3)
    v = np.concatenate([[0.0, 448.0, 449.0, 1.75, 3.4e38, 1e-45, 2.0 ** -96 * 448, 2.0 ** -96 * 449, np.inf, np.nan],
                        np.nextafter(np.float32(448) * np.float32(2) ** np.arange(-90, 100, 7, dtype=np.float32), np.float32(np.inf), dtype=np.float32),
                        np.float32(448) * np.float32(2) ** np.arange(-90, 100, 7, dtype=np.float32),
                        np.exp(rng.uniform(-80, 80, 300))]).astype(np.float32)
    out = subprocess.run([str(exe)], input="\n".join("%x" % u for u in v.view(np.uint32)), capture_output=True, text=True, check=True).stdout.split("\n")
    for a, line in zip(v, out):
        byte, inv, sc = (int(f, 16 if i else 10) for i, f in enumerate(line.split()))
        inv, sc = (np.array([u], np.uint32).view(np.float32)[0] for u in (inv, sc))
        if not np.isfinite(a):
            assert byte == 255 and np.isnan(inv) and np.isnan(sc)
            continue
        k = Q.exponents(np.array([[np.float64(a)]]))[0]
        assert byte == k + 127 and np.float64(sc) == 2.0 ** k and np.float64(inv) == 2.0 ** -k, (a, byte, k)
