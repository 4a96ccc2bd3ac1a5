"""How large tables may be for the calls that change them: so large that a step of a workgroup beyond the last entry still fits 32 bits (host only: every call here is
refused, or asks for sizes)."""
import ctypes as C

import pytest

from tests import test_cache_host as H
from tests import test_pages_host as P


@pytest.fixture(scope="module")
def B():
    from paper_2507_08143_amd import compactor
    return compactor


@pytest.mark.parametrize("nreq,table_len", [(2, (1 << 30) - 513), (3, 715827542), (7, 306783232), (16383, 131079)])
def test_entries_of_all_tables(B, nreq, table_len):
    n = C.c_size_t(0)
    most = (0x7fffffff - 1024) // nreq
    for size in (B._lib.compactor_pages_reserve_workspace_size, B._lib.compactor_pages_compact_workspace_size):
        for entries, code in ((table_len, B.OK if table_len <= most else B.EINVAL), (most, B.OK if most <= 1 << 30 else B.EINVAL), (most + 1, B.EINVAL)):
            cache = H._cache(B, nreq=nreq, page_size=1, table_len=entries, table_stride=entries)
            assert size(C.byref(cache), C.byref(n)) == code, entries
    cache = H._cache(B, nreq=nreq, page_size=1, table_len=most + 1, table_stride=most + 1)
    assert P._reserve(B, cache, P._params(B)) == B.EINVAL and P._compact(B, cache) == B.EINVAL
    assert B._lib.compactor_pages_fork(C.byref(cache), 0xa00000, 0xb00000, None) == B.EINVAL
    assert B._lib.compactor_pages_release(C.byref(cache), 0xa00000, 0, None) == B.EINVAL
