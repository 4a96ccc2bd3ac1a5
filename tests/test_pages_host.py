"""What the calls on pages refuse, found on the host before anything is enqueued (no GPU needed: the pointers are made up and every call
here is refused)."""
import ctypes as C

import pytest
import torch

from tests import test_cache_host as H
from tests import test_mx_host as M
from tests.test_cache_host import _g

WS = 0x1000000


@pytest.fixture(scope="module")
def B():
    from paper_2507_08143_amd import compactor
    return compactor


def _params(B, **kw):
    d = dict(refs=0xa00000, new_tokens=0, tokens=1, own_all=0, pairs=0xb00000, done=0xc00000)
    d.update(kw)
    return B._PagesReserve(**d)


def _ref(x):
    return C.byref(x) if x is not None else None


def _reserve(B, cache, params, ws=WS, wsb=1 << 40):
    return B._lib.compactor_pages_reserve(_ref(cache), _ref(params), ws, wsb, None)


def _compact(B, cache, refs=0xa00000, pairs=0xb00000, done=0xc00000, ws=WS, wsb=1 << 40):
    return B._lib.compactor_pages_compact(_ref(cache), refs, pairs, done, ws, wsb, None)


def _copies(B, pairs=0xb00000, most=10, done=0xc00000, cache=None, mx=None):
    return {B._lib.compactor_pages_copy(_ref(cache or H._cache(B)), pairs, most, done, None),
            B._lib.compactor_mx_pages_copy(_ref(mx or M._mx(B)), pairs, most, done, None)}


BAD = [(dict(nreq=0), "EINVAL"), (dict(nreq=16385), "EINVAL"), (dict(nreq=16384, table_len=1 << 18, table_stride=1 << 18), "EINVAL"), (dict(head_dim=64), "EUNSUPPORTED"),
       (dict(page_size=0), "EINVAL"), (dict(num_pages=0), "EINVAL"), (dict(num_pages=(1 << 30) + 1), "EINVAL"), (dict(table_len=0), "EINVAL"), (dict(tables=0), "EINVAL"), (dict(counts=0), "EINVAL"),
       (dict(count_stride_b=-1), "EINVAL"), (dict(tables=0x30002), "EALIGN"), (dict(counts=0x40001), "EALIGN"), (dict(seen=0x50002), "EALIGN")]


@pytest.mark.parametrize("kw,code", BAD, ids=[str(k) for k, _ in BAD])
def test_bad_caches(B, kw, code):
    cache = H._cache(B, **kw)
    code = getattr(B, code)
    assert _reserve(B, cache, _params(B)) == code and _compact(B, cache) == code
    assert B._lib.compactor_pages_fork(_ref(cache), 0xa00000, 0xb00000, None) == code
    assert B._lib.compactor_pages_release(_ref(cache), 0xa00000, 0, None) == code


def test_bad_arguments(B):
    cache = H._cache(B)
    assert _reserve(B, None, _params(B)) == B.EINVAL and _reserve(B, cache, None) == B.EINVAL and _compact(B, None) == B.EINVAL
    for kw, code in ((dict(refs=0), B.EINVAL), (dict(pairs=0), B.EINVAL), (dict(done=0), B.EINVAL), (dict(tokens=-1), B.EINVAL), (dict(refs=0xa00002), B.EALIGN),
                     (dict(pairs=0xb00004), B.EALIGN), (dict(done=0xc00002), B.EALIGN), (dict(new_tokens=0x2), B.EALIGN)):
        assert _reserve(B, cache, _params(B, **kw)) == code, kw
        kw = {k: v for k, v in kw.items() if k in ("refs", "pairs", "done")}
        if kw:
            assert _compact(B, cache, **kw) == code, kw
    for size, call in ((B._lib.compactor_pages_reserve_workspace_size, lambda **kw: _reserve(B, cache, _params(B), **kw)),
                       (B._lib.compactor_pages_compact_workspace_size, lambda **kw: _compact(B, cache, **kw))):
        n = C.c_size_t(0)
        assert size(_ref(cache), C.byref(n)) == 0 and n.value >= 400
        assert call(ws=0) == B.EWORKSPACE and call(wsb=n.value - 1) == B.EWORKSPACE and call(ws=WS + 16) == B.EALIGN
        assert size(_ref(cache), None) == B.EINVAL and size(None, C.byref(n)) == B.EINVAL and size(_ref(H._cache(B, nreq=16385)), C.byref(n)) == B.EINVAL
    for refs, parents, code in ((0, 0xb00000, B.EINVAL), (0xa00000, 0, B.EINVAL), (0xa00001, 0xb00000, B.EALIGN), (0xa00000, 0xb00002, B.EALIGN)):
        assert B._lib.compactor_pages_fork(_ref(cache), refs, parents, None) == code
    for refs, finished, code in ((0, 0, B.EINVAL), (0xa00001, 0, B.EALIGN), (0xa00000, 0xb00002, B.EALIGN)):
        assert B._lib.compactor_pages_release(_ref(cache), refs, finished, None) == code


def test_bad_copies(B):
    assert _copies(B, pairs=0) == {B.EINVAL} and _copies(B, most=0) == {B.EINVAL} and _copies(B, done=0) == {B.EINVAL}
    assert _copies(B, pairs=0xb00004) == {B.EALIGN} and _copies(B, done=0xc00002) == {B.EALIGN}
    for kw, code in ((dict(k_pages=0), B.EINVAL), (dict(slot_stride=16), B.EINVAL), (dict(page_stride=-16), B.EINVAL), (dict(k_pages=0x10008), B.EALIGN),
                     (dict(mass=0), B.EINVAL), (dict(mass=0x60002), B.EALIGN)):
        assert _copies(B, cache=H._cache(B, **kw), mx=M._mx(B, **kw)) == {code}, kw
    for layers in (8, 2):              # more than 2^30 units of 16 bytes a page, or numbers of its state
        huge = dict(page_size=1 << 20, kv_heads=1024, layers=layers, table_len=2, table_stride=2)
        assert _copies(B, cache=H._cache(B, **huge), mx=M._mx(B, **huge)) == {B.EINVAL}


def test_the_calls_check_their_tensors(B):
    i32 = torch.int32
    refs, three = _g(20, dtype=i32), _g(3, dtype=i32)
    for c, mx in ((H._handle(B), False), (M._handle(B), True)):
        copy, other = (B.compactor_mx_pages_copy, B.compactor_pages_copy) if mx else (B.compactor_pages_copy, B.compactor_mx_pages_copy)
        pairs, done = _g(15, 2, dtype=i32), _g(2, dtype=i32)
        for bad in (_g(19, dtype=i32), _g(20), _g(40, dtype=i32)[::2], _g(20, 1, dtype=i32)):
            for call in (lambda: B.compactor_pages_reserve(c, bad, 1), lambda: B.compactor_pages_fork(c, bad, three), lambda: B.compactor_pages_release(c, bad),
                         lambda: B.compactor_pages_compact(c, bad)):
                with pytest.raises(ValueError):
                    call()
        for call in (lambda: B.compactor_pages_reserve(c, refs, -1), lambda: B.compactor_pages_reserve(c, refs, 1 << 31),
                     lambda: B.compactor_pages_reserve(c, refs, 1, new_tokens=refs), lambda: B.compactor_pages_reserve(c, refs, 1, pairs=pairs[:14]),
                     lambda: B.compactor_pages_reserve(c, refs, 1, done=_g(3, dtype=i32)), lambda: B.compactor_pages_reserve(c, refs, 1, workspace=_g(3)),
                     lambda: B.compactor_pages_fork(c, refs, refs), lambda: B.compactor_pages_fork(c, refs, three.long()),
                     lambda: B.compactor_pages_release(c, refs, finished=three.bool()), lambda: B.compactor_pages_compact(c, refs, pairs=pairs),
                     lambda: B.compactor_pages_compact(c, refs, done=done.long()), lambda: copy(c, pairs.long(), done), lambda: copy(c, pairs[:, :1], done),
                     lambda: copy(c, pairs.flatten(), done), lambda: copy(c, pairs[:0], done), lambda: copy(c, pairs, done[:1]), lambda: other(c, pairs, done)):
            with pytest.raises(ValueError):
                call()
        part = c.layer(1)                              # shares its tables with the other layer
        for call in (lambda: B.compactor_pages_reserve(part, refs, 1), lambda: B.compactor_pages_fork(part, refs, three), lambda: B.compactor_pages_release(part, refs),
                     lambda: B.compactor_pages_compact(part, refs), lambda: copy(part, pairs, done), lambda: copy(part.layer(0), pairs, done)):
            with pytest.raises(ValueError):
                call()
        assert c.layer(0, 2)._whole


def test_struct_layouts_match_the_header(B):
    assert C.sizeof(B._PagesReserve) == 8 + 8 + 4 + 4 + 8 + 8
