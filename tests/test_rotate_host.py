"""What the calls that norm and rotate refuse, found on the host before anything is enqueued (no GPU needed: the pointers are made up
and every call here is refused)."""
import ctypes as C

import pytest
import torch

from tests import test_cache_host as H
from tests import test_mx_host as M
from tests.test_cache_host import _g, _rows


@pytest.fixture(scope="module")
def B():
    from paper_2507_08143_amd import compactor
    return compactor


def _rotation(B, **kw):
    d = dict(freqs=0x700000, rotary_dim=128, interleaved=0, q_norm=0x800000, k_norm=0x900000, eps=1e-6)
    d.update(kw)
    return B._Rotation(**d)


def _rotate(B, **kw):
    d = dict(q=0x100000, k=0x200000, q_out=0x300000, k_out=0x400000, k_plain=0x500000, positions=0x600000, position_stride_b=4, new_tokens=0,
             nreq=2, layers=1, tokens=4, q_heads=32, kv_heads=8)
    for n in ("q", "k", "q_out", "k_out", "k_plain"):
        d.update({n + "_stride_b": 65536, n + "_stride_l": 65536, n + "_stride_t": 4096, n + "_stride_h": 128})
    d.update(kw)
    return B._RotateRows(**d)


def _queries(B, **kw):
    d = dict(q=0x300000, q_out=0x400000, q_heads=32)
    for n in ("q", "q_out"):
        d.update({n + "_stride_b": 65536, n + "_stride_l": 65536, n + "_stride_t": 4096, n + "_stride_h": 128})
    d.update(kw)
    return B._RotateQueries(**d)


def _ref(x):
    return C.byref(x) if x is not None else None


BAD_ROTATIONS = [(dict(freqs=0), "EINVAL"), (dict(rotary_dim=0), "EUNSUPPORTED"), (dict(rotary_dim=130), "EUNSUPPORTED"), (dict(rotary_dim=136), "EUNSUPPORTED"),
                 (dict(rotary_dim=20), "EUNSUPPORTED"), (dict(rotary_dim=-8), "EUNSUPPORTED"), (dict(eps=0.0), "EINVAL"), (dict(eps=-1.0), "EINVAL"),
                 (dict(eps=float("nan")), "EINVAL"), (dict(eps=float("inf")), "EINVAL"), (dict(freqs=0x700004), "EALIGN"), (dict(q_norm=0x800004), "EALIGN"),
                 (dict(k_norm=0x900008), "EALIGN")]


def _appends(B, rotation, rows, queries, cache=None, mx=None):
    return {B._lib.compactor_cache_append_rotated(_ref(cache or H._cache(B)), _ref(rotation), _ref(rows), _ref(queries), None),
            B._lib.compactor_mx_append_rotated(_ref(mx or M._mx(B)), _ref(rotation), _ref(rows), _ref(queries), None)}


@pytest.mark.parametrize("kw,code", BAD_ROTATIONS, ids=[str(k) for k, _ in BAD_ROTATIONS])
def test_bad_rotations(B, kw, code):
    assert B._lib.compactor_rotate(_ref(_rotation(B, **kw)), _ref(_rotate(B)), None) == getattr(B, code)
    assert _appends(B, _rotation(B, **kw), _rows(B), _queries(B)) == {getattr(B, code)}


def test_bad_rows(B):
    assert B._lib.compactor_rotate(None, _ref(_rotate(B)), None) == B.EINVAL
    assert B._lib.compactor_rotate(_ref(_rotation(B)), None, None) == B.EINVAL
    for kw, code in ([(dict([(n, 0)]), B.EINVAL) for n in ("q", "k", "q_out", "k_out", "positions", "nreq", "layers", "tokens")] +
                     [(dict([(n, 0x1000008)]), B.EALIGN) for n in ("q", "k", "q_out", "k_out", "k_plain")] +
                     [(dict([(n + "_stride_" + d, -8)]), B.EINVAL) for n in ("q", "k", "q_out", "k_out", "k_plain") for d in "blth"] +
                     [(dict([(n + "_stride_" + d, 132)]), B.EALIGN) for n in ("q", "k", "q_out", "k_out", "k_plain") for d in "blth"] +
                     [(dict(q_heads=0, kv_heads=0), B.EINVAL), (dict(q_heads=(1 << 20) + 1), B.EINVAL), (dict(kv_heads=(1 << 20) + 1), B.EINVAL), (dict(q_heads=-1), B.EINVAL), (dict(kv_heads=-1), B.EINVAL),
                      (dict(position_stride_b=-1), B.EINVAL), (dict(positions=0x600002), B.EALIGN), (dict(new_tokens=0x2), B.EALIGN),
                      (dict(q_out=0x100000, q_out_stride_t=8192), B.EINVAL), (dict(k_out=0x200000, k_out_stride_h=256), B.EINVAL),
                      (dict(k_plain=0x200000, k_plain_stride_h=256), B.EINVAL), (dict(k_plain=0x400000), B.EINVAL), (dict(q_out=0x200000), B.EINVAL),
                      (dict(q_out=0x400000), B.EINVAL), (dict(q_out=0x500000), B.EINVAL), (dict(k_out=0x100000), B.EINVAL), (dict(k_plain=0x100000), B.EINVAL),
                      (dict(nreq=1 << 20, layers=1 << 12), B.EINVAL), (dict(nreq=1 << 20, tokens=1 << 12), B.EINVAL), (dict(nreq=1 << 24, tokens=16), B.EINVAL)]):
        assert B._lib.compactor_rotate(_ref(_rotation(B)), _ref(_rotate(B, **kw)), None) == code, kw


def test_bad_appends(B):
    rows, queries, rotation = _rows(B), _queries(B), _rotation(B)
    assert _appends(B, None, rows, queries) == {B.EINVAL}
    assert _appends(B, rotation, None, queries) == {B.EINVAL}
    for kw, code in ((dict(k=0), B.EINVAL), (dict(v=0), B.EINVAL), (dict(tokens=0), B.EINVAL), (dict(stride_t=-8), B.EINVAL), (dict(stride_h=4), B.EALIGN),
                     (dict(k=0x100008), B.EALIGN), (dict(v=0x200002), B.EALIGN), (dict(new_tokens=2), B.EALIGN)):
        assert _appends(B, rotation, _rows(B, **kw), queries) == {code}, kw
    for kw, code in ((dict(q=0), B.EINVAL), (dict(q_out=0), B.EINVAL), (dict(q_heads=0), B.EINVAL), (dict(q_heads=12), B.EINVAL), (dict(q_heads=4), B.EINVAL), (dict(q_heads=1 << 21), B.EINVAL),
                     (dict(q_stride_b=-8), B.EINVAL), (dict(q_out_stride_l=-8), B.EINVAL), (dict(q_stride_t=4), B.EALIGN), (dict(q_out_stride_h=12), B.EALIGN),
                     (dict(q=0x300008), B.EALIGN), (dict(q_out=0x400004), B.EALIGN), (dict(q_out=0x300000, q_out_stride_h=256), B.EINVAL)):
        assert _appends(B, rotation, rows, _queries(B, **kw)) == {code}, kw
    bare = dict(seen=0, mass=0, positions=0)          # the positions are what the cache has seen
    assert _appends(B, rotation, rows, queries, H._cache(B, **bare), M._mx(B, **bare)) == {B.EINVAL}
    wide = dict(nreq=1 << 26)
    assert _appends(B, rotation, rows, queries, H._cache(B, **wide), M._mx(B, **wide)) == {B.EINVAL}


def _made(B, **kw):
    d = dict(freqs=_g(64, dtype=torch.float64), q_norm=_g(2, 128), k_norm=_g(2, 128))
    d.update(kw)
    return B.Rotation(**d)


def test_the_rotation_checks_its_tensors(B):
    r = _made(B)
    assert (r.rotary_dim, r.layers) == (128, 2) and r.layer(1)._c.q_norm == r._c.q_norm + 512
    assert _made(B, q_norm=None, k_norm=None).layer(7).layers is None and _made(B, freqs=_g(16, dtype=torch.float64)).rotary_dim == 32
    for kw in (dict(freqs=_g(64)), dict(freqs=_g(63, dtype=torch.float64)), dict(freqs=_g(128, dtype=torch.float64)[::2]), dict(rotary_dim=64),
               dict(freqs=_g(0, dtype=torch.float64)), dict(q_norm=_g(128)), dict(q_norm=_g(3, 128)), dict(k_norm=_g(2, 64)), dict(k_norm=_g(2, 256)[:, ::2]),
               dict(k_norm=_g(2, 128, dtype=torch.float64)), dict(freqs=torch.zeros(64, dtype=torch.float64), q_norm=None, k_norm=None)):
        with pytest.raises(ValueError):
            _made(B, **kw)
    with pytest.raises(ValueError):
        r.layer(2)


def test_the_calls_check_their_tensors(B):
    r = _made(B)
    bf = torch.bfloat16
    q, k, pos = _g(3, 2, 5, 8, 128, dtype=bf), _g(3, 2, 5, 4, 128, dtype=bf), _g(3, 5, dtype=torch.int32)
    for a, kw in (((None, None, pos), {}), ((_g(3, 2, 5, 8, 128), k, pos), {}), ((q[0], k, pos), {}), ((q, k[:, :1], pos), {}), ((q[..., :64], k, pos), {}),
                  ((q[:, :1], k[:, :1], pos), {}), ((q, k, pos[:2]), {}), ((q, k, pos.long()), {}), ((q, k, _g(5, 3, dtype=torch.int32).t()), {}),
                  ((q, k, pos), dict(new_tokens=_g(2, dtype=torch.int32))), ((q, k, pos), dict(new_tokens=_g(3))), ((q, k, pos), dict(q_out=k)),
                  ((q, k, pos), dict(k_out=_g(3, 2, 5, 4, 128))), ((q, k, pos), dict(k_plain=k[:, :, :1].expand(3, 2, 5, 4, 128))),
                  ((q, None, pos), dict(want_plain=True)), ((q, None, pos), dict(k_out=k)), ((None, k, pos), dict(q_out=q))):
        with pytest.raises(ValueError):
            B.compactor_rotate(r, *a, **kw)
    plain, mx = H._handle(B), M._handle(B)
    for call, c, other in ((B.compactor_cache_append_rotated, plain, mx), (B.compactor_mx_append_rotated, mx, plain)):
        for a, kw in (((other, r, k, k), {}), ((c, r.layer(0), k, k), {}), ((c, r, k, k, q[:, :, :4]), {}), ((c, r, k, k, _g(3, 2, 5, 8, 128)), {}),
                      ((c, r, k[:2], k[:2]), {}), ((c, r, k, k), dict(q_out=q)), ((c, r, k, k, q), dict(q_out=k)),
                      ((c, r, k, k, q), dict(new_tokens=_g(2, dtype=torch.int32)))):
            with pytest.raises(ValueError):
                call(*a, **kw)


def test_struct_layouts_match_the_header(B):
    assert C.sizeof(B._Rotation) == 8 + 4 + 4 + 8 + 8 + 8
    assert C.sizeof(B._RotateRows) == 5 * 8 + 20 * 8 + 3 * 8 + 5 * 4 + 4 and C.sizeof(B._RotateQueries) == 2 * 8 + 8 * 8 + 8
