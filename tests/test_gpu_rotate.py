"""Norms and rotation of queries and keys against the float64 oracle, and the appends that rotate against rotate and append."""
import numpy as np
import pytest
import torch

from oracle import rotate_oracle as R
from tests import cache_util as U
from tests import gpu_util as GU
from tests import mx_util as X
from tests.test_gpu_cache import DEV, _counts, _new

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(scope="module")
def C():
    return GU.binding()


def _rotation(C, rotary=128, interleaved=False, q_norm=True, k_norm=True, layers=1, seed=1, base=500000.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    freqs = base ** (-torch.arange(rotary // 2, device=DEV, dtype=torch.float64) / (rotary // 2))
    w = [0.5 + torch.rand(layers, 128, generator=g, device=DEV) if on else None for on in (q_norm, k_norm)]
    return C.Rotation(freqs, rotary, interleaved, *w, EPS)


def _rows(shape, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    t = torch.randn(shape, generator=g, device=DEV)
    t[..., 3] *= 20
    return (t * torch.exp(2 * torch.randn((*shape[:-1], 1), generator=g, device=DEV))).to(torch.bfloat16)


def _want(rotation, x, weight, positions):
    """-> (y, rotated, how far they may be off).  With u = 2^-24: a sum of 128 squares is off by 128 u relative, its root by half of that, the
    reciprocal root, the two products and eps by 6 u: y by 70 u.  Sine and cosine are off by 6 u (their argument by 2, of a size of
    up to 1, the series by 4 in all), a product and a sum by 2: (|a| + |b|) 80 u.  Then one rounding to bf16."""
    x = U.f64(x)
    w = None if weight is None else weight.double().cpu().numpy()[None, :, None, None, :]
    y = R.norm(x, w, EPS)
    f = rotation.freqs.cpu().numpy()
    z = R.rotate(y, positions[:, None, :, None], f, rotation.rotary_dim, rotation.interleaved)
    n, u = rotation.rotary_dim, U.STEP32
    size = np.abs(y).copy()
    if rotation.interleaved:
        pair = np.abs(y[..., :n:2]) + np.abs(y[..., 1:n:2])
        size[..., :n:2], size[..., 1:n:2] = pair, pair
    else:
        pair = np.abs(y[..., :n // 2]) + np.abs(y[..., n // 2:n])
        size[..., :n // 2], size[..., n // 2:n] = pair, pair
    ey, ez = 70 * u * np.abs(y), 80 * u * size
    return y, z, U.STEP16 * (np.abs(y) + ey) + ey + 2.0 ** -133, U.STEP16 * (np.abs(z) + ez) + ez + 2.0 ** -133


def _near(got, want, bound, what):
    err = np.abs(U.f64(got) - want)
    assert np.all(err <= bound), "%s: off by %.3g of %.3g allowed" % (what, err.max(), bound.reshape(-1)[np.argmax(err - bound)])


def _positions(B, T, far, seed=3):
    g = torch.Generator().manual_seed(seed)
    return (torch.randint(0, far + 1, (B, 1), generator=g) + torch.arange(T)).to(torch.int32)


def _check(C, rotation, q, k, positions, what=""):
    pos = positions.to(torch.float64).numpy()
    got_q, got_k, plain = C.compactor_rotate(rotation, q, k, positions.to(DEV), want_plain=k is not None)
    if q is not None:
        _, z, _, bz = _want(rotation, q, rotation.q_norm, pos)
        _near(got_q, z, bz, what + " q")
    if k is not None:
        y, z, by, bz = _want(rotation, k, rotation.k_norm, pos)
        _near(got_k, z, bz, what + " k")
        if rotation.k_norm is None:
            assert torch.equal(U.bits(plain), U.bits(k))
        _near(plain, y, by, what + " plain")
    return got_q, got_k, plain


@pytest.mark.parametrize("rotary", [128, 64, 32, 96, 8, 72, 120, 16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("q_norm,k_norm", [(True, True), (False, False), (True, False), (False, True)])
def test_rotate(C, rotary, interleaved, q_norm, k_norm):
    rotation = _rotation(C, rotary, interleaved, q_norm, k_norm, layers=2)
    _check(C, rotation, _rows((2, 2, 5, 12, 128), 1), _rows((2, 2, 5, 3, 128), 2), _positions(2, 5, 1000))


@pytest.mark.parametrize("B,L,T,Hq,H", [(1, 1, 1, 1, 1), (1, 1, 1, 7, 1), (1, 1, 1, 64, 8), (3, 1, 1, 28, 4), (1, 1, 700, 32, 8), (2, 3, 333, 5, 5),
                                        (1, 1, 4097, 9, 3), (1, 1, 2, 0, 4), (1, 1, 3, 6, 0), (40, 2, 60, 4, 1), (1, 1, 1, 300, 2)])
def test_rotate_shapes(C, B, L, T, Hq, H):
    q = _rows((B, L, T, Hq, 128), 3) if Hq else None
    k = _rows((B, L, T, H, 128), 4) if H else None
    _check(C, _rotation(C, layers=L), q, k, _positions(B, T, 100000))


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotate_far_and_negative_positions(C, interleaved):
    """The angle is taken modulo 2 pi without loss: its distance from the oracle's does not grow with it."""
    positions = torch.tensor([[0, 1, -1, 2 ** 20, 2 ** 24 + 1, -2 ** 24 - 1, 2 ** 31 - 1, -2 ** 31, 123456789, 710, 355, 103993]], dtype=torch.int32)
    rotation = _rotation(C, interleaved=interleaved, base=3.0)
    _check(C, rotation, _rows((1, 1, 12, 3, 128), 5), _rows((1, 1, 12, 2, 128), 6), positions)
    one = C.compactor_rotate(rotation, _rows((3, 1, 12, 3, 128), 5), None, positions[0].to(DEV))[0]          # the same for all requests
    two = C.compactor_rotate(rotation, _rows((3, 1, 12, 3, 128), 5), None, positions.expand(3, 12).to(DEV))[0]
    assert torch.equal(U.bits(one), U.bits(two))


def test_rotate_numbers_that_are_none(C):
    """They stay in their pair without a norm, in their row with one."""
    q = _rows((1, 1, 1, 4, 128), 7)
    q[0, 0, 0, 0, 5], q[0, 0, 0, 1, 100], q[0, 0, 0, 2, 127] = float("nan"), float("inf"), float("nan")
    q[0, 0, 0, 3, 120] = -float("inf")
    got = C.compactor_rotate(_rotation(C, 96, q_norm=False), q, None, torch.tensor([5], dtype=torch.int32, device=DEV))[0][0, 0, 0]
    bad = torch.zeros(4, 128, dtype=torch.bool, device=DEV)
    bad[0, 5] = bad[0, 53] = bad[1, 100] = bad[2, 127] = bad[3, 120] = True
    assert torch.equal(~torch.isfinite(got.float()), bad) and float(got[1, 100]) == float("inf") and float(got[3, 120]) == -float("inf")
    got = C.compactor_rotate(_rotation(C, 96), q, None, torch.tensor([5], dtype=torch.int32, device=DEV))[0][0, 0, 0].float()
    assert torch.isnan(got[0]).all() and torch.isnan(got[2]).all() and torch.isnan(got[1, 100]) and not got[1, :100].any()
    zero = torch.zeros(1, 1, 1, 2, 128, dtype=torch.bfloat16, device=DEV)
    assert not C.compactor_rotate(_rotation(C), zero, None, torch.tensor([5], dtype=torch.int32, device=DEV))[0].any()


def test_rotate_padding_strides_and_in_place(C):
    rotation = _rotation(C, 64, layers=2)
    big = _rows((2, 2, 9, 20, 160), 8)                                     # [layer, request, token, q k and v heads, channel]
    q, k = big[..., :12, 16:144].permute(1, 0, 2, 3, 4), big[..., 12:16, 16:144].permute(1, 0, 2, 3, 4)
    positions, new = _positions(2, 9, 5000).to(DEV), torch.tensor([4, 30], dtype=torch.int32, device=DEV)
    want_q, want_k, want_plain = C.compactor_rotate(rotation, q.contiguous(), k.contiguous(), positions, want_plain=True)
    outs = [torch.full(t.shape, 9.0, dtype=torch.bfloat16, device=DEV).transpose(2, 3).contiguous().transpose(2, 3) for t in (q, k, k)]
    C.compactor_rotate(rotation, q, k, positions, new_tokens=new, q_out=outs[0], k_out=outs[1], k_plain=outs[2])
    for t, w in zip(outs, (want_q, want_k, want_plain)):
        assert torch.equal(t[0, :, :4], w[0, :, :4]) and torch.equal(t[1], w[1]) and bool((t[0, :, 4:] == 9.0).all())
    was = big.clone()
    plain = torch.empty_like(want_k)
    C.compactor_rotate(rotation, q, k, positions, new_tokens=new, q_out=q, k_out=k, k_plain=plain)
    assert torch.equal(q[0, :, :4], want_q[0, :, :4]) and torch.equal(k[1], want_k[1]) and torch.equal(plain[1], want_plain[1])
    big[:, 0, :4, :16, 16:144], big[:, 1, :, :16, 16:144] = was[:, 0, :4, :16, 16:144], was[:, 1, :, :16, 16:144]
    assert torch.equal(U.bits(big), U.bits(was))
    one = rotation.layer(1)
    assert torch.equal(C.compactor_rotate(one, q[:, 1:2].contiguous(), None, positions)[0], want_q[:, 1:2])


# ------------------------------------------------------------------------------------------ append
class _Twins:
    """Two caches that hold the same, of 16 bits or of 4."""

    def __init__(self, C, mx, counts, **kw):
        make = X.Paged if mx else U.Paged
        self.mx, self.a, self.b = mx, make(C, DEV, counts, **kw), make(C, DEV, counts, **kw)

    def cache(self, P):
        return P.mx_handle() if self.mx else P.handle()

    def same(self, what=""):
        (X.same if self.mx else U.same_pool)(self.a, self.b.snapshot(), what=what)


def _separately(C, P, cache, rotation, q, k, v, new):
    """rotate, then append; the heads of a layer may have seen different numbers of tokens."""
    B, L, T, H, _ = k.shape
    rotated_q, rotated_k = torch.full_like(q, 9.0), torch.empty_like(k)
    for h in range(H):
        for l in range(L):
            positions = (P.seen[:, l, h:h + 1] + torch.arange(T, device=DEV)).to(torch.int32)
            G = q.shape[3] // H
            a, b, _ = C.compactor_rotate(rotation.layer(l), q[:, l:l + 1, :, h * G:(h + 1) * G], k[:, l:l + 1, :, h:h + 1], positions)
            n = torch.full((B,), T) if new is None else torch.tensor(new).clamp(0, T)
            real = (torch.arange(T) < n.view(B, 1)).to(DEV).view(B, T, 1, 1)
            rotated_q[:, l, :, h * G:(h + 1) * G] = torch.where(real, a[:, 0], rotated_q[:, l, :, h * G:(h + 1) * G])
            rotated_k[:, l, :, h] = b[:, 0, :, 0]
    (C.compactor_mx_append if isinstance(cache, C.MxCache) else C.compactor_cache_append)(cache, rotated_k, v, new_tokens=_new(new))
    return rotated_q


def _together(C, cache):
    return C.compactor_mx_append_rotated if isinstance(cache, C.MxCache) else C.compactor_cache_append_rotated


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("T,new", [(1, None), (1, [1, 0, 1]), (2, None), (5, [5, 0, 3]), (9, None), (64, [64, -1, 70]), (65, [0, 65, 64]), (130, [130, 3, 129])])
@pytest.mark.parametrize("G,rotary,interleaved,page,layout", [(1, 128, False, 16, "token"), (4, 64, True, 24, "head"), (7, 96, False, 7, "layer"),
                                                              (16, 32, True, 64, "head"), (2, 8, False, 16, "token")])
def test_append_rotated(C, mx, T, new, G, rotary, interleaved, page, layout):
    twins = _Twins(C, mx, _counts(3, 2, 3, 40, 0, 17, 33, 100), page=page, layout=layout, room=90)          # not room for all
    for P in (twins.a, twins.b):
        P.tables[1, (40 + T // 2) // page] = -1
        P.seen.copy_((torch.arange(18) * 1000).view(3, 2, 3))
    rotation = _rotation(C, rotary, interleaved, q_norm=G != 4, k_norm=G != 7, layers=2)
    q, k, v = _rows((3, 2, T, 3 * G, 128), 1), _rows((3, 2, T, 3, 128), 2), _rows((3, 2, T, 3, 128), 3)
    a, b = twins.cache(twins.a), twins.cache(twins.b)
    want = _separately(C, twins.b, b, rotation, q, k, v, new)
    got = _together(C, a)(a, rotation, k, v, q, new_tokens=_new(new), q_out=torch.full_like(q, 9.0))
    assert torch.equal(U.bits(got), U.bits(want))
    twins.same("T %d" % T)
    # without queries, in place, and one layer
    _separately(C, twins.b, b, rotation, q, k, v, new)
    assert _together(C, a)(a, rotation, k, v, new_tokens=_new(new)) is None
    twins.same("without queries")
    qq = q.clone()
    one = a.layer(1)
    before = twins.a.counts.clone()
    _together(C, a)(one, rotation.layer(1), k[:, 1:], v[:, 1:], qq[:, 1:], new_tokens=_new(new), q_out=qq[:, 1:])
    assert torch.equal(qq[:, 0], q[:, 0]) and torch.equal(twins.a.counts[:, 0], before[:, 0])


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("B,L,H,G,T", [(1, 1, 1, 1, 1), (67, 1, 3, 4, 1), (5, 7, 9, 5, 1), (130, 1, 8, 2, 1), (33, 1, 5, 3, 2), (300, 1, 1, 8, 1),
                                       (3, 1, 2, 7, 8), (3, 1, 2, 7, 9), (40, 2, 8, 2, 20), (64, 4, 8, 1, 48), (64, 8, 8, 1, 60), (64, 8, 8, 1, 70)])
def test_append_rotated_shapes(C, mx, B, L, H, G, T):
    twins = _Twins(C, mx, _counts(B, L, H, 5, 0, 17, 33), page=16, room=max(8, T - 3))
    rotation = _rotation(C, layers=L)
    q, k, v = _rows((B, L, T, H * G, 128), 1), _rows((B, L, T, H, 128), 2), _rows((B, L, T, H, 128), 3)
    for P in (twins.a, twins.b):
        P.seen.copy_(P.seen[:, :1, :1].expand(P.seen.shape).contiguous())
    a, b = twins.cache(twins.a), twins.cache(twins.b)
    positions = (twins.b.seen[:, 0, :1] + torch.arange(T, device=DEV)).to(torch.int32)
    want, rk, _ = C.compactor_rotate(rotation, q, k, positions)
    (C.compactor_mx_append if mx else C.compactor_cache_append)(b, rk, v)
    got = _together(C, a)(a, rotation, k, v, q)
    assert torch.equal(U.bits(got), U.bits(want))
    twins.same()


@pytest.mark.parametrize("mx", [False, True])
def test_a_captured_step(C, mx):
    """Keys rotated into the cache, queries rotated in place, attention: replayed as the cache grows, against the eager calls on a copy, on
    a stream of its own."""
    twins = _Twins(C, mx, _counts(3, 1, 4, 100, 90, 33, 140), page=16, room=80)
    rotation = _rotation(C)
    k, v = (torch.empty(3, 1, 1, 4, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    q = torch.empty(3, 1, 1, 16, 128, dtype=torch.bfloat16, device=DEV)
    new = torch.ones(3, dtype=torch.int32, device=DEV)
    a, b = twins.cache(twins.a), twins.cache(twins.b)
    attend = C.compactor_mx_attention if mx else C.compactor_cache_attention

    def step(cache, stream=None):
        rotated = torch.zeros_like(q)
        _together(C, cache)(cache, rotation, k, v, q, new_tokens=new, q_out=rotated, stream=stream)
        return rotated, attend(cache, rotated, new_tokens=new, accumulate=True, stream=stream)[0]

    for t in (k, v, q):
        t.normal_()
    step(twins.cache((X.Paged if mx else U.Paged)(C, DEV, _counts(3, 1, 4, 100, 90, 33, 140), page=16, room=80)))
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        got = step(a)
    g = torch.Generator(device=DEV)
    g.manual_seed(7)
    for i in range(6):
        for t in (k, v, q):
            t.copy_(torch.randn(t.shape, generator=g, device=DEV))
        new.copy_(torch.tensor([1, i % 2, 1 if i < 3 else 0], dtype=torch.int32))
        graph.replay()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            want = step(b, side)
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(U.bits(x), U.bits(y)), i
        twins.same("replay %d" % i)
