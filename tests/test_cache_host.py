"""What the serving calls refuse, found on the host before anything is enqueued (no GPU needed: the pointers are made up
and every call here is refused)."""
import ctypes as C

import pytest
import torch


@pytest.fixture(scope="module")
def B():
    from paper_2507_08143_amd import compactor
    return compactor


def _cache(B, **kw):
    pool = dict(k_pages=0x10000, v_pages=0x20000, page_stride=16 * 8 * 128, layer_stride=0, head_stride=128,
                slot_stride=8 * 128, page_size=16, num_pages=100)
    c = dict(tables=0x30000, table_stride=10, table_len=10, nreq=2, layers=1, kv_heads=8, head_dim=128, counts=0x40000,
             seen=0x50000, count_stride_b=8, count_stride_l=8, mass=0x60000, positions=0x70000, state_page_stride=128,
             state_layer_stride=128, state_head_stride=16)
    for n, v in kw.items():
        (pool if n in pool else c)[n] = v
    return B._Cache(pool=B._PagePool(**pool), **c)


def _rows(B, **kw):
    d = dict(k=0x100000, v=0x200000, stride_b=1024, stride_l=1024, stride_t=1024, stride_h=128, new_tokens=0, tokens=1)
    d.update(kw)
    return B._CacheRows(**d)


def _query(B, **kw):
    d = dict(q=0x100000, out=0x200000, lse=0, q_stride_b=4096, q_stride_l=4096, q_stride_t=4096, q_stride_h=128,
             out_stride_b=4096, out_stride_l=4096, out_stride_t=4096, out_stride_h=128, new_tokens=0, tokens=1, q_heads=32,
             scale=0.0, softcap=0.0, accumulate=0, max_tokens=0)
    d.update(kw)
    return B._CacheQuery(**d)


def _evict(B, **kw):
    d = dict(budget=5, budgets=0, sink=0, recent=0, scope=0, max_tokens=0)
    d.update(kw)
    return B._CacheEvict(**d)


def _append(B, cache, rows):
    return B._lib.compactor_cache_append(C.byref(cache) if cache else None, C.byref(rows) if rows else None, None)


def _attend(B, cache, query, ws=0x1000000, wsb=0):
    return B._lib.compactor_cache_attention(C.byref(cache), C.byref(query) if query else None, ws, wsb, None)


def _evicts(B, cache, evict, ws=0x1000000, wsb=0):
    return B._lib.compactor_cache_evict(C.byref(cache), C.byref(evict) if evict else None, ws, wsb, None)


BAD_CACHES = [
    (dict(nreq=0), "EINVAL"), (dict(layers=0), "EINVAL"), (dict(kv_heads=-1), "EINVAL"), (dict(head_dim=64), "EUNSUPPORTED"),
    (dict(layers=1 << 11, kv_heads=1 << 10), "EINVAL"), (dict(nreq=1 << 30, kv_heads=4), "EINVAL"),
    (dict(page_size=0), "EINVAL"), (dict(num_pages=0), "EINVAL"), (dict(table_len=0), "EINVAL"), (dict(table_stride=9), "EINVAL"),
    (dict(table_len=1 << 20, table_stride=1 << 20, page_size=1 << 11), "EINVAL"),
    (dict(table_len=(1 << 20) + 1, table_stride=1 << 21, page_size=1 << 10), "EINVAL"),
    (dict(k_pages=0), "EINVAL"), (dict(v_pages=0), "EINVAL"), (dict(tables=0), "EINVAL"), (dict(counts=0), "EINVAL"),
    (dict(slot_stride=64), "EINVAL"), (dict(page_stride=-8), "EINVAL"), (dict(count_stride_b=-1), "EINVAL"),
    (dict(state_page_stride=-1), "EINVAL"), (dict(seen=0), "EINVAL"), (dict(mass=0), "EINVAL"), (dict(positions=0), "EINVAL"),
    (dict(k_pages=0x10008), "EALIGN"), (dict(head_stride=132), "EALIGN"), (dict(tables=0x30002), "EALIGN"),
    (dict(mass=0x60001), "EALIGN"),
]


@pytest.mark.parametrize("kw,code", BAD_CACHES, ids=[str(k) for k, _ in BAD_CACHES])
def test_bad_caches(B, kw, code):
    cache, code = _cache(B, **kw), getattr(B, code)
    assert _append(B, cache, _rows(B)) == code
    assert _attend(B, cache, _query(B)) == code
    assert _evicts(B, cache, _evict(B)) == code
    p = B._Params(int(cache.layers), int(cache.kv_heads), 128, 48, 0, 0.0, 0.3, 0, 0, 0, 0, None)
    reqs = (B._Request * 2)(*[B._Request(0, 0, 0, 0, 0, 0, 128, 100, 0.5)] * 2)
    if code == B.EINVAL and 1 <= cache.layers * cache.kv_heads <= 1 << 20 and cache.kv_heads > 0:
        assert B._lib.compactor_cache_admit(C.byref(p), reqs, 2, 0x1000, 0x2000, 0, C.byref(cache), None) == code


def test_a_cache_without_state(B):
    bare = _cache(B, seen=0, mass=0, positions=0)
    assert _evicts(B, bare, _evict(B)) == B.EINVAL
    assert _attend(B, bare, _query(B, accumulate=1)) == B.EINVAL
    n = C.c_size_t(7)
    assert B._lib.compactor_cache_attention_workspace_size(C.byref(bare), C.byref(_query(B)), C.byref(n)) == 0


def test_bad_rows(B):
    cache = _cache(B)
    assert _append(B, None, _rows(B)) == B.EINVAL
    assert _append(B, cache, None) == B.EINVAL
    for kw, code in ((dict(k=0), B.EINVAL), (dict(v=0), B.EINVAL), (dict(tokens=0), B.EINVAL), (dict(stride_t=-8), B.EINVAL),
                     (dict(stride_h=4), B.EALIGN), (dict(k=0x100004), B.EALIGN), (dict(new_tokens=2), B.EALIGN)):
        assert _append(B, cache, _rows(B, **kw)) == code, kw


def test_bad_queries(B):
    cache = _cache(B)
    assert _attend(B, cache, None) == B.EINVAL
    for kw, code in ((dict(q=0), B.EINVAL), (dict(out=0), B.EINVAL), (dict(tokens=0), B.EINVAL), (dict(q_heads=7), B.EINVAL),
                     (dict(q_heads=12), B.EINVAL), (dict(tokens=17), B.EUNSUPPORTED), (dict(q_heads=520), B.EUNSUPPORTED),
                     (dict(scale=-1.0), B.EINVAL), (dict(scale=float("nan")), B.EINVAL), (dict(scale=float("inf")), B.EINVAL),
                     (dict(softcap=-1.0), B.EINVAL), (dict(softcap=float("inf")), B.EINVAL), (dict(max_tokens=-1), B.EINVAL),
                     (dict(scale=3e38), B.EINVAL), (dict(softcap=3e38), B.EINVAL), (dict(scale=1.0, softcap=1e-39), B.EINVAL),
                     (dict(q_stride_t=-8), B.EINVAL), (dict(out_stride_h=-128), B.EINVAL), (dict(q=0x100002), B.EALIGN),
                     (dict(out=0x200008), B.EALIGN), (dict(out_stride_h=4), B.EALIGN), (dict(q_stride_b=12), B.EALIGN),
                     (dict(lse=0x3), B.EALIGN), (dict(new_tokens=0x6), B.EALIGN)):
        assert _attend(B, cache, _query(B, **kw)) == code, kw
    q = _query(B, accumulate=1)
    n = C.c_size_t(0)
    assert B._lib.compactor_cache_attention_workspace_size(C.byref(cache), C.byref(q), C.byref(n)) == 0
    assert n.value >= 2 * 8 * 4 * 160 * 4          # heads, query heads of each, slots, fp32
    assert _attend(B, cache, q, ws=0, wsb=n.value) == B.EWORKSPACE
    assert _attend(B, cache, q, wsb=n.value - 1) == B.EWORKSPACE
    assert _attend(B, cache, q, ws=0x1000010, wsb=n.value) == B.EALIGN
    assert B._lib.compactor_cache_attention_workspace_size(C.byref(cache), C.byref(q), None) == B.EINVAL
    assert B._lib.compactor_cache_attention_workspace_size(C.byref(cache), None, C.byref(n)) == B.EINVAL


def test_attention_does_not_write_over_its_queries(B):
    """They are read again, for the weights of many rows."""
    assert _attend(B, _cache(B), _query(B, out=0x100000)) == B.EINVAL


def test_the_workspace_follows_max_tokens(B):
    sizes = []
    for most in (1, 50, 160, 1000, 0):
        q, n = _query(B, accumulate=1, max_tokens=most), C.c_size_t(0)
        assert B._lib.compactor_cache_attention_workspace_size(C.byref(_cache(B)), C.byref(q), C.byref(n)) == 0
        sizes.append(n.value)
    assert sizes == sorted(sizes) and sizes[2] == sizes[3] == sizes[4]
    # a head alone needs none up to 16384 tokens, nor a layer of 8 heads up to 2048 each
    for scope, tokens, some in ((0, (10, 16384), False), (0, (16385, 40000, 0), True), (1, (10, 2048), False), (1, (2049, 9000, 0), True)):
        n = [C.c_size_t(7) for _ in tokens]
        for out, most in zip(n, tokens):
            e = _evict(B, max_tokens=most, scope=scope)
            cache = _cache(B, table_len=4000, table_stride=4000)
            assert B._lib.compactor_cache_evict_workspace_size(C.byref(cache), C.byref(e), C.byref(out)) == 0
        sizes = [x.value for x in n]
        assert sizes == sorted(sizes) and (sizes[0] > 0 and len(set(sizes)) == len(sizes) if some else set(sizes) == {0})


@pytest.mark.parametrize("G,room", [(40, 1024), (64, 256), (64, 1024)])
def test_no_workspace_for_a_join_of_heads_of_one_workgroup(B, G, room):
    """Weights of many rows of many short heads: room for a weight a slot, a sum a row and what is known of a head, and for no partial outputs."""
    heads = 16384
    cache = _cache(B, nreq=heads // 8, table_len=room // 16, table_stride=room // 16)
    q, n = _query(B, accumulate=1, q_heads=8 * G), C.c_size_t(0)
    assert B._lib.compactor_cache_attention_workspace_size(C.byref(cache), C.byref(q), C.byref(n)) == 0
    least = heads * (4 * room + 8 * G)
    assert least <= n.value <= least + 64 * heads


def test_calls_that_no_launch_can_take(B):
    """2^32 threads or more: refused before anything is enqueued, not by a launch that fails."""
    def cache(heads, **kw):
        return _cache(B, nreq=heads // 8, **kw)

    assert _append(B, cache(1 << 28), _rows(B)) == B.EINVAL
    assert _append(B, cache(1 << 28), _rows(B, tokens=8)) == B.EINVAL
    assert _append(B, cache(1 << 24), _rows(B, tokens=64)) == B.EINVAL
    assert _append(B, cache(1 << 20), _rows(B, tokens=1024)) == B.EINVAL
    assert _attend(B, cache(1 << 24), _query(B)) == B.EINVAL
    assert _attend(B, cache(1 << 24, table_len=1000, table_stride=1000), _query(B)) == B.EINVAL
    assert _evicts(B, cache(1 << 22), _evict(B)) == B.EINVAL
    assert _evicts(B, cache(1 << 25), _evict(B, scope=1)) == B.EINVAL
    assert _evicts(B, cache(1 << 20, table_len=2048, table_stride=2048), _evict(B), wsb=1 << 60) == B.EINVAL


def test_bad_evictions(B):
    cache, n = _cache(B, table_len=300, table_stride=300), C.c_size_t(0)
    assert B._lib.compactor_cache_evict_workspace_size(C.byref(cache), C.byref(_evict(B, scope=1)), C.byref(n)) == 0 and n.value > 0
    assert _evicts(B, cache, None) == B.EINVAL
    for kw in (dict(budget=-1), dict(sink=-1), dict(recent=-1), dict(scope=2), dict(max_tokens=-5)):
        assert _evicts(B, cache, _evict(B, **kw), wsb=n.value) == B.EINVAL, kw
    assert _evicts(B, cache, _evict(B, budgets=0x2), wsb=n.value) == B.EALIGN
    assert _evicts(B, cache, _evict(B, scope=1), ws=0, wsb=n.value) == B.EWORKSPACE
    assert _evicts(B, cache, _evict(B, scope=1), wsb=n.value - 1) == B.EWORKSPACE
    assert _evicts(B, cache, _evict(B, scope=1), ws=0x1000080, wsb=n.value) == B.EALIGN
    wide = _cache(B, table_len=1 << 20, table_stride=1 << 20, kv_heads=256)
    assert _evicts(B, wide, _evict(B, scope=1), wsb=1 << 50) == B.EINVAL


def test_admission_needs_the_cache_of_the_call(B):
    cache = _cache(B)
    p = B._Params(1, 8, 128, 48, 0, 0.0, 0.3, 0, 0, 0, 0, None)
    reqs = (B._Request * 2)(*[B._Request(0, 0, 0, 0, 0, 0, 128, 100, 0.5)] * 2)

    def admit(p=p, n=2, idx=0x1000, cnt=0x2000, cache=cache):
        return B._lib.compactor_cache_admit(C.byref(p), reqs, n, idx, cnt, 0, C.byref(cache) if cache else None, None)

    assert admit(idx=0) == B.EINVAL
    assert admit(cnt=0) == B.EINVAL
    assert admit(cache=None) == B.EINVAL
    assert admit(n=1) == B.EINVAL
    assert admit(p=B._Params(1, 4, 128, 48, 0, 0.0, 0.3, 0, 0, 0, 0, None)) == B.EINVAL
    assert admit(p=B._Params(2, 8, 128, 48, 0, 0.0, 0.3, 0, 0, 0, 0, None)) == B.EINVAL
    reqs[1].n = 0
    assert admit() == B.EINVAL


class _Gpu(torch.Tensor):
    """A CPU tensor that says it lives on a GPU: only its shape, type and strides are looked at here."""
    is_cuda = True


def _g(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(_Gpu)


def _handle(B, P=20, L=2, S=16, H=4, R=3, N=5, **kw):
    d = dict(k_pages=_g(P, L, S, H, 128, dtype=torch.bfloat16), v_pages=_g(P, L, S, H, 128, dtype=torch.bfloat16),
             tables=_g(R, N, dtype=torch.int32), counts=_g(R, L, H, dtype=torch.int32), seen=_g(R, L, H, dtype=torch.int32),
             mass=_g(P, L, H, S), positions=_g(P, L, H, S, dtype=torch.int32))
    d.update(kw)
    return B.Cache(**d)


def test_the_handle_checks_its_tensors(B):
    c = _handle(B)
    assert (c.nreq, c.layers, c.kv_heads) == (3, 2, 4)
    assert c._c.table_len == 5 and c._c.pool.num_pages == 20 and c._c.pool.page_size == 16
    one = c.layer(1)
    assert one.layers == 1 and one._c.pool.k_pages == c._c.pool.k_pages + 16 * 4 * 128 * 2
    assert one._c.counts == c._c.counts + 16 and one._c.mass == c._c.mass + 4 * 4 * 16
    assert _handle(B, tables=_g(1, 5, dtype=torch.int32).expand(3, 5)[:1], counts=_g(1, 2, 4, dtype=torch.int32),
                   seen=_g(1, 2, 4, dtype=torch.int32)).nreq == 1
    for kw in (dict(k_pages=_g(20, 2, 16, 4, 128)), dict(v_pages=_g(20, 2, 16, 5, 128, dtype=torch.bfloat16)),
               dict(v_pages=_g(20, 2, 4, 16, 128, dtype=torch.bfloat16).transpose(2, 3)), dict(tables=_g(3, 5)),
               dict(tables=_g(3, dtype=torch.int32)), dict(tables=_g(3, 0, dtype=torch.int32)),
               dict(tables=_g(1, 5, dtype=torch.int32).expand(3, 5)), dict(tables=_g(5, 3, dtype=torch.int32).t()),
               dict(counts=_g(3, 2, 4)), dict(counts=_g(3, 2, 5, dtype=torch.int32)), dict(seen=_g(3, 4, 2, dtype=torch.int32).transpose(1, 2)),
               dict(seen=None), dict(mass=None), dict(positions=None), dict(seen=None, positions=None),
               dict(mass=_g(20, 2, 16, 4)), dict(mass=_g(20, 2, 4, 16, dtype=torch.float16)),
               dict(positions=_g(20, 2, 4, 16)), dict(counts=_g(1, 2, 4, dtype=torch.int32).expand(3, 2, 4),
                                                      seen=_g(1, 2, 4, dtype=torch.int32).expand(3, 2, 4)),
               dict(counts=torch.zeros(3, 2, 4, dtype=torch.int32)),
               dict(k_pages=_g(20, 1, 16, 4, 128, dtype=torch.bfloat16).expand(20, 2, 16, 4, 128),
                    v_pages=_g(20, 1, 16, 4, 128, dtype=torch.bfloat16).expand(20, 2, 16, 4, 128))):
        with pytest.raises(ValueError):
            _handle(B, **kw)
    with pytest.raises(ValueError):
        c.layer(2)


def test_the_calls_check_their_tensors(B):
    c = _handle(B)
    k = _g(3, 2, 1, 4, 128, dtype=torch.bfloat16)
    for bad in ((k[:2], k[:2]), (k, k.expand(3, 2, 1, 4, 128).contiguous()[..., :64]), (_g(3, 2, 1, 4, 128), k), (k[0], k[0]),
                (k, _g(3, 2, 4, 1, 128, dtype=torch.bfloat16).transpose(2, 3)[:, :, :, ::1][:, :1])):
        with pytest.raises(ValueError):
            B.compactor_cache_append(c, *bad)
    for new in (_g(2, dtype=torch.int32), _g(3), _g(6, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError):
            B.compactor_cache_append(c, k, k, new_tokens=new)
        with pytest.raises(ValueError):
            B.compactor_cache_attention(c, k, new_tokens=new)
    q = _g(3, 2, 1, 8, 128, dtype=torch.bfloat16)
    for bad in (_g(3, 2, 1, 8, 128), q[:, :1], q[0], _g(3, 2, 1, 128, 8, dtype=torch.bfloat16).transpose(3, 4)):
        with pytest.raises(ValueError):
            B.compactor_cache_attention(c, bad)
    for kw in (dict(out=_g(3, 2, 1, 8, 128)), dict(out=q[:, :, :, :4]), dict(out=q[:, :, :, :1].expand(3, 2, 1, 8, 128)),
               dict(lse=_g(47)), dict(lse=_g(48, dtype=torch.float64)), dict(workspace=_g(100))):
        with pytest.raises(ValueError):
            B.compactor_cache_attention(c, q, **kw)
    for kw in (dict(), dict(budget=3, budgets=_g(3, dtype=torch.int32)), dict(budgets=_g(2, dtype=torch.int32)),
               dict(budgets=_g(3)), dict(budget=3, workspace=_g(100))):
        with pytest.raises(ValueError):
            B.compactor_cache_evict(c, **kw)
    p = B.Params(2, 4)
    some = torch.zeros(1, 1, 1, 128, dtype=torch.bfloat16)
    reqs = [B.Request(k_score=some.expand(2, 4, 10, 128), v_cache=some.expand(2, 4, 10, 128), ratio=0.5) for _ in range(3)]
    idx, cnt = _g(3 * 8 * 5, dtype=torch.int32), _g(24, dtype=torch.int32)
    for a in ((p, reqs[:2], idx, cnt), (p, reqs, idx[1:], cnt), (p, reqs, idx, cnt[1:]), (p, reqs, _g(120), cnt),
              (B.Params(1, 8), reqs, idx, cnt)):
        with pytest.raises(ValueError):
            B.compactor_cache_admit(*a, c)
    with pytest.raises(ValueError):
        B.compactor_cache_admit(p, reqs, idx, cnt, c, scores=_g(239))


def test_numbers_that_do_not_fit_the_structures(B):
    """A budget of 2^32 is not one of 0, and tokens protected without end are not unprotected."""
    c = _handle(B)
    q, k = _g(3, 2, 1, 8, 128, dtype=torch.bfloat16), _g(3, 2, 1, 4, 128, dtype=torch.bfloat16)
    for x in (1 << 31, 1 << 32, (1 << 32) + 5, 1 << 63, -1):
        for kw in (dict(budget=x), dict(budget=3, sink=x), dict(budget=3, recent=x), dict(budget=3, max_tokens=x)):
            with pytest.raises(ValueError):
                B.compactor_cache_evict(c, **kw)
        with pytest.raises(ValueError):
            B.compactor_cache_attention(c, q, max_tokens=x)
        with pytest.raises(ValueError):
            B.compactor_cache_attention_workspace_size(c, q, max_tokens=x)
        with pytest.raises(ValueError):
            B.compactor_cache_evict_workspace_size(c, max_tokens=x)
    with pytest.raises(ValueError):
        B.compactor_cache_append(c, *[k.expand(3, 2, (1 << 32) + 1, 4, 128)] * 2)
