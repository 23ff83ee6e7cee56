"""8-bit paged cache, host side: the limits that the header states."""
import ctypes

import pytest

from paper_2603_30033_b200 import binding as Bd
from paper_2603_30033_b200 import build as Bu
from tests.test_q8_cpu import append, cache, desc, read, store


@pytest.fixture(scope="module")
def lib():
    Bu.build()
    return Bd.load_library()


def test_widest_rows(lib):
    for call in (append, store, read):
        assert call(lib, d=desc(r=(2, 16, 1282))) == call(lib, d=desc(t=(2, 16, 1281))) == -2
        assert call(lib, d=desc(r=(2, 16, 1280), t=(2, 16, 1280)), T=0) != -2


def test_append_workspace_by_tokens(lib):
    """Shapes that go through fp32 rows need room for them; those of the tensor cores do not."""
    need = lambda d, T: lib.tucker_cache_append_paged_q8_workspace_bytes(ctypes.byref(d), ctypes.byref(cache()), T)
    for d in (desc(), desc(dtype=Bd.TA_DTYPE_BF16)):
        assert need(d, 100000) >= 4 * 100000 * 32
    fast = desc(d_model=4096, n_H=32, r=(2, 128, 128), t=(2, 128, 128), dtype=Bd.TA_DTYPE_BF16)
    assert need(fast, 1 << 20) < 16 << 20
