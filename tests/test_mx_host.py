"""What the calls of a cache in 4 bits refuse, found on the host before anything is enqueued (no GPU needed: the pointers are made
up and every call here is refused)."""
import ctypes as C

import pytest
import torch

from tests import test_cache_host as H
from tests.test_cache_host import _evict, _g, _query, _rows


@pytest.fixture(scope="module")
def B():
    from paper_2507_08143_amd import compactor
    return compactor


def _mx(B, k_scales=0x80000, v_scales=0x90000, **kw):
    kw = {"page_stride": 16 * 8 * 64, "head_stride": 64, "slot_stride": 8 * 64, **kw}
    return B._MxCache(H._cache(B, **kw), k_scales, v_scales)


def _read(B, **kw):
    d = dict(k=0x100000, v=0x200000, stride_b=1024, stride_l=1024, stride_t=1024, stride_h=128, new_tokens=0, tokens=1, first=0)
    d.update(kw)
    return B._CacheRowsOut(**d)


def _ref(x):
    return C.byref(x) if x is not None else None


def _calls(B, cache, source=None):
    return {"append": B._lib.compactor_mx_append(_ref(cache), _ref(_rows(B)), None),
            "read": B._lib.compactor_mx_read(_ref(cache), _ref(_read(B)), None),
            "store": B._lib.compactor_mx_store(_ref(cache), _ref(source or H._cache(B, k_pages=0x110000, v_pages=0x120000, counts=0x130000)), None),
            "attention": B._lib.compactor_mx_attention(_ref(cache), _ref(_query(B)), 0x1000000, 0, None),
            "evict": B._lib.compactor_mx_evict(_ref(cache), _ref(_evict(B)), 0x1000000, 0, None)}


BAD = [(dict(nreq=0), "EINVAL"), (dict(head_dim=64), "EUNSUPPORTED"), (dict(page_size=0), "EINVAL"), (dict(table_len=0), "EINVAL"),
       (dict(k_pages=0), "EINVAL"), (dict(tables=0), "EINVAL"), (dict(counts=0), "EINVAL"), (dict(k_scales=0), "EINVAL"), (dict(v_scales=0), "EINVAL"),
       (dict(slot_stride=48), "EINVAL"), (dict(page_stride=-16), "EINVAL"), (dict(state_head_stride=-1), "EINVAL"), (dict(mass=0), "EINVAL"),
       (dict(k_pages=0x10008), "EALIGN"), (dict(head_stride=72), "EALIGN"), (dict(page_stride=8), "EALIGN"), (dict(k_scales=0x80002), "EALIGN"),
       (dict(v_scales=0x90001), "EALIGN"), (dict(positions=0x70002), "EALIGN"), (dict(counts=0x40001), "EALIGN"), (dict(seen=0x50002), "EALIGN")]


@pytest.mark.parametrize("kw,code", BAD, ids=[str(k) for k, _ in BAD])
def test_bad_caches(B, kw, code):
    for name, got in _calls(B, _mx(B, **kw)).items():
        assert got == getattr(B, code), name


def test_no_cache(B):
    assert set(_calls(B, None).values()) == {B.EINVAL}


def test_a_cache_without_state(B):
    bare = _mx(B, seen=0, mass=0, positions=0)
    assert B._lib.compactor_mx_evict(C.byref(bare), C.byref(_evict(B)), 0x1000000, 0, None) == B.EINVAL
    assert B._lib.compactor_mx_attention(C.byref(bare), C.byref(_query(B, accumulate=1)), 0x1000000, 1 << 40, None) == B.EINVAL


def test_bad_sources(B):
    good = dict(k_pages=0x110000, v_pages=0x120000, counts=0x130000)
    for kw in (dict(nreq=3), dict(layers=2), dict(kv_heads=4), dict(seen=0, mass=0, positions=0), dict(counts=0x40000), dict(k_pages=0x10000),
               dict(v_pages=0x20000), dict(k_pages=0x20000), dict(v_pages=0x10000), dict(k_pages=0), dict(tables=0)):
        assert _calls(B, _mx(B), H._cache(B, **{**good, **kw}))["store"] == B.EINVAL, kw
    assert B._lib.compactor_mx_store(C.byref(_mx(B)), None, None) == B.EINVAL
    assert _calls(B, _mx(B), H._cache(B, **{**good, "k_pages": 0x110008}))["store"] == B.EALIGN


def test_bad_reads(B):
    for kw, code in ((dict(k=0), B.EINVAL), (dict(v=0), B.EINVAL), (dict(v=0x100000), B.EINVAL), (dict(tokens=0), B.EINVAL), (dict(first=-2), B.EINVAL),
                     (dict(stride_t=-8), B.EINVAL), (dict(stride_h=4), B.EALIGN), (dict(k=0x100008), B.EALIGN), (dict(new_tokens=2), B.EALIGN)):
        assert B._lib.compactor_mx_read(C.byref(_mx(B)), C.byref(_read(B, **kw)), None) == code, kw
    assert B._lib.compactor_mx_read(C.byref(_mx(B)), None, None) == B.EINVAL


def test_bad_rows_queries_and_evictions(B):
    cache, n = _mx(B), C.c_size_t(0)
    for kw, code in ((dict(k=0), B.EINVAL), (dict(tokens=0), B.EINVAL), (dict(stride_h=4), B.EALIGN)):
        assert B._lib.compactor_mx_append(C.byref(cache), C.byref(_rows(B, **kw)), None) == code
    for kw, code in ((dict(q=0), B.EINVAL), (dict(out=0x100000), B.EINVAL), (dict(q_heads=12), B.EINVAL), (dict(tokens=17), B.EUNSUPPORTED),
                     (dict(softcap=-1.0), B.EINVAL), (dict(out_stride_h=4), B.EALIGN)):
        assert B._lib.compactor_mx_attention(C.byref(cache), C.byref(_query(B, **kw)), 0x1000000, 0, None) == code
    q = _query(B, accumulate=1)
    assert B._lib.compactor_mx_attention_workspace_size(C.byref(cache), C.byref(q), C.byref(n)) == 0 and n.value > 0
    assert B._lib.compactor_mx_attention(C.byref(cache), C.byref(q), 0x1000000, n.value - 1, None) == B.EWORKSPACE
    assert B._lib.compactor_mx_attention(C.byref(cache), C.byref(q), 0x1000010, n.value, None) == B.EALIGN
    assert B._lib.compactor_mx_evict(C.byref(cache), C.byref(_evict(B, budget=-1)), 0x1000000, 0, None) == B.EINVAL
    long = _mx(B, table_len=300, table_stride=300)
    assert B._lib.compactor_mx_evict_workspace_size(C.byref(long), C.byref(_evict(B, scope=1)), C.byref(n)) == 0 and n.value > 0
    assert B._lib.compactor_mx_evict(C.byref(long), C.byref(_evict(B, scope=1)), 0x1000000, n.value - 1, None) == B.EWORKSPACE
    assert B._lib.compactor_mx_attention_workspace_size(None, C.byref(q), C.byref(n)) == B.EINVAL
    assert B._lib.compactor_mx_evict_workspace_size(None, C.byref(_evict(B)), C.byref(n)) == B.EINVAL


def test_calls_that_no_launch_can_take(B):
    wide = _mx(B, nreq=1 << 25)
    assert set(_calls(B, wide, H._cache(B, nreq=1 << 25, k_pages=0x110000, v_pages=0x120000, counts=0x130000)).values()) == {B.EINVAL}
    assert B._lib.compactor_mx_read(C.byref(_mx(B, nreq=1 << 12)), C.byref(_read(B, tokens=1 << 22)), None) == B.EINVAL


def _handle(B, P=20, L=2, S=16, H=4, R=3, N=5, **kw):
    u8 = torch.uint8
    d = dict(k_pages=_g(P, L, S, H, 64, dtype=u8), v_pages=_g(P, L, S, H, 64, dtype=u8), k_scales=_g(P, L, H, S, 4, dtype=u8),
             v_scales=_g(P, L, H, S, 4, dtype=u8), tables=_g(R, N, dtype=torch.int32), counts=_g(R, L, H, dtype=torch.int32),
             seen=_g(R, L, H, dtype=torch.int32), mass=_g(P, L, H, S), positions=_g(P, L, H, S, dtype=torch.int32))
    d.update(kw)
    return B.MxCache(**d)


def test_the_handle_checks_its_tensors(B):
    c = _handle(B)
    assert (c.nreq, c.layers, c.kv_heads) == (3, 2, 4) and c._c.pool.slot_stride == 256 and c._c.state_page_stride == 128
    one = c.layer(1)
    assert one.layers == 1 and one._c.pool.k_pages == c._c.pool.k_pages + 16 * 4 * 64 and one._mx.k_scales == c._mx.k_scales + 4 * 4 * 16
    bare = _handle(B, seen=None, mass=None, positions=None)
    assert bare._c.state_page_stride == 128 and bare._c.mass is None
    u8 = torch.uint8
    for kw in (dict(k_pages=_g(20, 2, 16, 4, 64)), dict(k_pages=_g(20, 2, 16, 4, 128, dtype=u8), v_pages=_g(20, 2, 16, 4, 128, dtype=u8)),
               dict(v_pages=_g(20, 2, 4, 16, 64, dtype=u8).transpose(2, 3)), dict(k_scales=_g(20, 2, 4, 16, 4)), dict(v_scales=_g(20, 2, 4, 16, dtype=u8)),
               dict(v_scales=_g(20, 2, 16, 4, 4, dtype=u8).transpose(2, 3)),
               dict(k_scales=_g(20, 2, 4, 16, 8, dtype=u8)[..., :4], v_scales=_g(20, 2, 4, 16, 8, dtype=u8)[..., :4]),
               dict(k_scales=_g(20, 2, 4, 17, 4, dtype=u8)[:, :, :, :16], v_scales=_g(20, 2, 4, 17, 4, dtype=u8)[:, :, :, :16]),
               dict(k_scales=_g(1, 2, 4, 16, 4, dtype=u8).expand(20, 2, 4, 16, 4), v_scales=_g(1, 2, 4, 16, 4, dtype=u8).expand(20, 2, 4, 16, 4)),
               dict(k_scales=torch.zeros(20, 2, 4, 16, 4, dtype=u8), v_scales=torch.zeros(20, 2, 4, 16, 4, dtype=u8)),
               dict(seen=None), dict(counts=_g(3, 2, 4)), dict(tables=_g(3, 5))):
        with pytest.raises(ValueError):
            _handle(B, **kw)


def test_calls_of_one_kind_refuse_the_other(B):
    mx, plain = _handle(B), H._handle(B)
    k = _g(3, 2, 1, 4, 128, dtype=torch.bfloat16)
    for call in (lambda: B.compactor_cache_append(mx, k, k), lambda: B.compactor_cache_attention(mx, k), lambda: B.compactor_cache_evict(mx, budget=3),
                 lambda: B.compactor_cache_attention_workspace_size(mx, k), lambda: B.compactor_cache_evict_workspace_size(mx),
                 lambda: B.compactor_mx_append(plain, k, k), lambda: B.compactor_mx_attention(plain, k), lambda: B.compactor_mx_evict(plain, budget=3),
                 lambda: B.compactor_mx_attention_workspace_size(plain, k), lambda: B.compactor_mx_evict_workspace_size(plain),
                 lambda: B.compactor_mx_read(plain, 3), lambda: B.compactor_mx_store(plain, plain), lambda: B.compactor_mx_store(mx, mx)):
        with pytest.raises(ValueError):
            call()


def test_the_calls_check_their_tensors(B):
    c = _handle(B)
    k = _g(3, 2, 4, 4, 128, dtype=torch.bfloat16)
    for kw in (dict(tokens=5, k=k, v=k.clone()), dict(tokens=4, k=k), dict(tokens=4, k=k, v=_g(3, 2, 4, 4, 128)), dict(tokens=-1), dict(tokens=1 << 31),
               dict(tokens=4, first=-1), dict(tokens=4, first=1 << 32), dict(tokens=4, k=k[:, :, :1].expand(3, 2, 4, 4, 128), v=k[:, :, :1].expand(3, 2, 4, 4, 128)),
               dict(tokens=4, k=k, v=k.clone(), new_tokens=_g(2, dtype=torch.int32))):
        with pytest.raises(ValueError):
            B.compactor_mx_read(c, **kw)
    with pytest.raises(ValueError):
        B.compactor_mx_store(c, H._handle(B, R=2))
    with pytest.raises(ValueError):
        B.compactor_mx_store(c, H._handle(B, seen=None, mass=None, positions=None))
    for bad in (_g(3, 2, 1, 4, 128), _g(3, 2, 1, 4, 64, dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            B.compactor_mx_append(c, bad, bad)
        with pytest.raises(ValueError):
            B.compactor_mx_attention(c, bad)


def test_struct_layouts_match_the_header(B):
    assert C.sizeof(B._MxCache) == C.sizeof(B._Cache) + 16 and C.sizeof(B._CacheRowsOut) == 2 * 8 + 4 * 8 + 8 + 8
