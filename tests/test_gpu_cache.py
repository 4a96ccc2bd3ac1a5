"""Serving from a paged cache against the float64 oracle: append, attention, eviction, admission, alone and together."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as O
from tests import cache_util as U
from tests import gpu_util as GU

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def C():
    return GU.binding()


def _queries(P, T, Hq, seed=5, gain=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (gain * torch.randn(P.B, P.L, T, Hq, 128, generator=g, device=DEV)).to(torch.bfloat16)


def _new(values):
    return None if values is None else torch.tensor(values, dtype=torch.int32, device=DEV)


def _attend(C, P, q, new=None, scale=0.0, cap=0.0, accumulate=True, most=0, what="", **kw):
    before = P.snapshot()
    out, lse = C.compactor_cache_attention(P.cache, q, new_tokens=_new(new), scale=scale, softcap=cap, accumulate=accumulate,
                                           max_tokens=most, want_lse=True, **kw)
    torch.cuda.synchronize()
    for n in ("k", "v"):
        assert torch.equal(U.bits(getattr(P, n)), U.bits(before[n])), what
    for n in ("counts", "seen", "positions"):
        assert torch.equal(getattr(P, n), before[n]), what
    if not accumulate:
        assert torch.equal(P.mass.view(torch.int32), before["mass"].view(torch.int32)), what
    U.check_attention(P, q, new, scale or 128 ** -0.5, cap, out, lse, before, accumulate, most, what)
    return out, lse


def _counts(B, L, H, *values):
    """Nested [B][L][H] counts that go round `values`."""
    it = 0
    got = []
    for _ in range(B):
        got.append([])
        for _ in range(L):
            got[-1].append([values[(it + h) % len(values)] for h in range(H)])
            it += H
    return got


# ------------------------------------------------------------------------------------------ attention
# lengths around every size that a tile, a wave or a page may have, an empty head among them
@pytest.mark.parametrize("page,layout", [(16, "token"), (32, "head"), (64, "layer"), (7, "token"), (24, "head"), (1, "token"),
                                         (128, "layer"), (8, "head"), (48, "token"), (1000, "head")])
@pytest.mark.parametrize("G", [1, 4])
def test_attention_lengths(C, page, layout, G):
    counts = _counts(3, 1, 8, 0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 511, 513, 700, 1023, 1025)
    P = U.Paged(C, DEV, counts, page=page, layout=layout, gain=8.0)
    _attend(C, P, _queries(P, 1, 8 * G), what="page %d" % page)


@pytest.mark.parametrize("G,T", [(1, 1), (2, 1), (3, 1), (5, 1), (7, 1), (8, 1), (16, 1), (17, 1), (32, 1), (64, 1), (33, 1),
                                 (1, 2), (4, 4), (4, 5), (8, 8), (5, 3), (1, 64), (2, 17), (3, 21)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_attention_rows(C, G, T, accumulate):
    counts = _counts(2, 2, 2, 333, 80, 64, 1, 0, 40, 129, 500)
    P = U.Paged(C, DEV, counts, page=16, layout="token", seed=G * 100 + T)
    _attend(C, P, _queries(P, T, 2 * G), accumulate=accumulate, what="G %d T %d" % (G, T))
    new = [T // 2, T + 5] if T > 1 else [0, 1]
    _attend(C, P, _queries(P, T, 2 * G), new=new, accumulate=accumulate, what="G %d T %d, padded" % (G, T))
    _attend(C, P, _queries(P, T, 2 * G), new=[-3, 1], accumulate=accumulate, what="G %d T %d, one token" % (G, T))


@pytest.mark.parametrize("scale,cap,gain", [(0.0, 30.0, 1.0), (0.5, 5.0, 8.0), (0.02, 0.0, 8.0), (1.0, 0.0, 20.0), (1.0, 50.0, 20.0),
                                            (0.0, 1e4, 1.0), (0.3, 4e6, 8.0), (0.0, 2e38, 1.0), (0.0, 0.01, 1.0), (1.0, 1e-30, 1.0)])
def test_attention_scales_and_caps(C, scale, cap, gain):
    """Large logits too: one slot that takes all the weight, caps that saturate, and caps that no logit comes near."""
    P = U.Paged(C, DEV, _counts(2, 1, 4, 700, 33, 5, 1500), page=16, gain=gain)
    _attend(C, P, _queries(P, 2, 16), scale=scale, cap=cap)


@pytest.mark.parametrize("B,L,H,n,page", [(1, 1, 1, 20011, 16), (1, 1, 4, 9001, 64), (2, 1, 1, 33000, 24), (1, 3, 2, 6007, 32),
                                          (1, 1, 2, 70001, 256)])
@pytest.mark.parametrize("G,T", [(4, 1), (7, 1), (5, 4)])
def test_attention_long(C, B, L, H, n, page, G, T):
    """Few heads whose length is shared by many workgroups, a short one beside them."""
    counts = _counts(B, L, H, n, n - 3 * page - 1, 5)
    P = U.Paged(C, DEV, counts, page=page, layout="head")
    _attend(C, P, _queries(P, T, H * G), cap=20.0 if T > 1 else 0.0)


@pytest.mark.parametrize("H,lengths,page", [(2, (9001, 300, 0, 1), 64), (1, (20011, 6000, 4500, 31), 24), (3, (5000, 3, 2500), 16), (1, (2100,) * 4, 7)])
@pytest.mark.parametrize("G,T", [(8, 5), (8, 8), (64, 1), (1, 33), (7, 7)])
@pytest.mark.parametrize("room", [0, 2 ** 28 + 1])
def test_attention_weights_of_many_rows(C, H, lengths, page, G, T, room):
    """More than 32 query rows over heads that several workgroups share, heads of one workgroup and empty ones beside them, padded
    requests, a page that is not there, capped or not; tables with room for `room` bytes of logits too."""
    P = U.Paged(C, DEV, _counts(4, 1, H, *lengths), page=page)
    P.tables[1, 1] = -1
    if room:             # (the oracle keeps to the pages that are there)
        wide = torch.full((4, room // (4 * H * G * T * page * 4) + 1), -1, dtype=torch.int32, device=DEV)
        wide[:, :P.per] = P.tables
        P.cache = C.Cache(P.k, P.v, wide, P.counts, P.seen, P.mass, P.positions)
        assert C.compactor_cache_attention_workspace_size(P.cache, _queries(P, T, H * G), accumulate=True) < 2 ** 28
    cap = 15.0 if T == 5 else 0.0
    _attend(C, P, _queries(P, T, H * G), cap=cap)
    _attend(C, P, _queries(P, T, H * G), new=[T - 1, 0, T, 1], cap=cap, most=9000 if H == 2 else 0)


def test_attention_weights_of_many_rows_of_many_short_heads(C):
    """The same where every head has a workgroup of its own."""
    P = U.Paged(C, DEV, _counts(20, 1, 55, 0, 1, 33, 40), page=16)
    wide = torch.full((20, 64), -1, dtype=torch.int32, device=DEV)
    wide[:, :P.per] = P.tables
    P.cache = C.Cache(P.k, P.v, wide, P.counts, P.seen, P.mass, P.positions)
    assert C.compactor_cache_attention_workspace_size(P.cache, _queries(P, 1, 55 * 64), accumulate=True) < 2 ** 28
    _attend(C, P, _queries(P, 1, 55 * 64), new=[1, 0] * 10)


@pytest.mark.parametrize("page", [16, 24])
@pytest.mark.parametrize("T", [1, 9])
def test_attention_of_one_long_request_among_many(C, page, T):
    """Few parts a head, because there are many heads: a wave has more tiles than it keeps places for."""
    P = U.Paged(C, DEV, [[[34001, 40, 0, 20000, 33999, 1, 128, 16385]]], page=page)
    B = 66
    tables = torch.full((B, P.per), -1, dtype=torch.int32, device=DEV)
    tables[0] = P.tables[0]
    counts, seen = (torch.zeros(B, 1, 8, dtype=torch.int32, device=DEV) for _ in range(2))
    counts[0] = P.counts[0]
    cache = C.Cache(P.k, P.v, tables, counts, seen, P.mass, P.positions)
    q = torch.zeros(B, 1, T, 32, 128, dtype=torch.bfloat16, device=DEV)
    q[:1] = _queries(P, T, 32)
    before = P.snapshot()
    out, lse = C.compactor_cache_attention(cache, q, accumulate=True, want_lse=True)
    torch.cuda.synchronize()
    assert not out[1:].float().any() and torch.isneginf(lse[1:]).all()
    U.check_attention(P, q[:1], None, 128 ** -0.5, 0.0, out[:1], lse[:1], before, True)


@pytest.mark.parametrize("B,L,H,lengths", [(5, 2, 9, (2000, 1, 0, 1025, 700, 128, 129, 1999)), (16, 1, 8, (1300,)), (16, 1, 8, (1290, 1300, 1280)),
                                           (43, 1, 7, (1100, 30, 0, 1500)), (37, 2, 4, (1100, 1090)), (8, 8, 8, (1030, 1024, 513, 60)),
                                           (65, 1, 8, (1100, 5, 900, 0, 1400)), (9, 8, 9, (1200,)), (1, 513, 1, (1025,)), (200, 3, 7, (40, 1100, 0))])
def test_attention_of_many_heads(C, B, L, H, lengths):
    """Heads of one length and of many, up to and beyond the number whose lengths a workgroup looks through."""
    P = U.Paged(C, DEV, _counts(B, L, H, *lengths), page=32, layout="token", seed=B)
    new = None if B % 2 else [b % 3 for b in range(B)]
    _attend(C, P, _queries(P, 2, H), new=new, accumulate=B != 37, what="%d heads" % (B * L * H))


@pytest.mark.parametrize("page", [16, 24, 128])
@pytest.mark.parametrize("fill", [float("nan"), float("inf"), -float("inf")])
def test_attention_does_not_look_past_the_end(C, page, fill):
    """Slots that no token is in, pages that nobody names, and pages that are not there hold anything."""
    counts = _counts(2, 1, 4, 0, 1, 45, 100, 300, 31, 33, 250)
    P = U.Paged(C, DEV, counts, page=page, room=60, fill=fill)
    P.tables[1, 1] = -1
    P.tables[0, 0] = P.pages + 7
    _attend(C, P, _queries(P, 3, 12))
    _attend(C, P, _queries(P, 3, 12), new=[2, 1], accumulate=False)


@pytest.mark.parametrize("fill", [float("nan"), float("inf"), 3e38])
@pytest.mark.parametrize("count,T", [(40, 4), (33, 2), (64, 5), (3, 5), (130, 7), (18, 16)])
def test_attention_does_not_look_ahead(C, fill, count, T):
    """The rows of later tokens, keys and values, do not reach the earlier ones."""
    P = U.Paged(C, DEV, _counts(1, 1, 2, count, count), page=16)
    q = _queries(P, T, 4)
    for h in range(2):
        s = count - 1                                  # seen by the last token alone
        p, a = int(P.tables[0, s // 16]), s % 16
        P.v[p, 0, a, h] = fill
        if h == 0:
            P.k[p, 0, a, h] = fill
    out, lse = C.compactor_cache_attention(P.cache, q, accumulate=True, want_lse=True)
    torch.cuda.synchronize()
    # All but the last token against the oracle, which does not look at the slot.  (Not against a run that finds a number in it: that
    # one multiplies the rows of later tokens in another order and with its weights in 16 bits, which the bounds allow for.)
    qd, od, ld = U.f64(q), U.f64(out), lse.double().cpu().numpy()
    for h in range(2):
        k, v, _, _, there = P.head(0, 0, h)
        for t, see in enumerate(O.sees(count, T, T)[:T - 1]):
            for g in range(2):
                row = (0, 0, t, 2 * h + g)
                want, want_lse, p = O.attend(qd[row], k, v, see, there, 128 ** -0.5, 0.0)
                b_out, b_lse, _ = U.attention_bounds(qd[row], k, v, see, there, 128 ** -0.5, 0.0, want, p)
                assert np.all(np.abs(od[row] - want) <= b_out), (h, t)
                assert ld[row] == want_lse or abs(ld[row] - want_lse) <= b_lse, (h, t)


def test_attention_values_that_are_seen_count(C):
    """What a query does see is not hidden: NaN and infinities come out as the formula has them."""
    P = U.Paged(C, DEV, _counts(1, 1, 3, 50, 50, 50), page=16)
    for h, x in ((0, float("nan")), (1, float("inf"))):
        P.v[int(P.tables[0, 1]), 0, 3, h, 7] = x
    P.k[int(P.tables[0, 0]), 0, 2, 2] = float("nan")
    out, lse = C.compactor_cache_attention(P.cache, _queries(P, 1, 6), want_lse=True)
    o = out[0, 0, 0].float()
    assert torch.isnan(o[0:2, 7]).all() and torch.isinf(o[2:4, 7]).all()
    rest = [c for c in range(128) if c != 7]
    assert torch.isfinite(o[0:4][:, rest]).all()
    assert torch.isnan(o[4:6]).all() and torch.isnan(lse[0, 0, 0, 4:6]).all()


@pytest.mark.parametrize("count,G,T", [(1, 1, 1), (1, 4, 1), (40, 4, 1), (129, 7, 1), (127, 4, 5), (100, 6, 6), (120, 8, 8), (2001, 4, 1)])
@pytest.mark.parametrize("page,gain", [(16, 1.0), (24, 8.0)])
def test_attention_infinite_values_that_are_seen(C, count, G, T, page, gain):
    """An infinity in channel s of the value of slot s: the infinity, of its sign, whatever the weight, and numbers elsewhere."""
    P = U.Paged(C, DEV, [[[count]]], page=page, gain=gain)
    n = min(count, 128) - T + 1                   # seen by all queries
    for s in range(n):
        P.v[int(P.tables[0, s // page]), 0, s % page, 0, s] = float("inf") if s % 3 else -float("inf")
    out, lse = C.compactor_cache_attention(P.cache, _queries(P, T, G), want_lse=True)
    o = out.float()
    want = torch.full((n,), float("inf"), device=DEV)
    want[::3] = -float("inf")
    assert torch.equal(o[..., :n], want.expand(1, 1, T, G, n)) and bool(torch.isfinite(o[..., n:]).all() & torch.isfinite(lse).all())


def _room_for_logits(C, P, G, T):
    """Tables so long that the logits of more than 32 rows would take more than 256 MB."""
    wide = torch.full((P.B, 2 ** 28 // (4 * P.B * P.L * P.H * G * T * P.page) + 2), -1, dtype=torch.int32, device=DEV)
    wide[:, :P.per] = P.tables
    P.cache = C.Cache(P.k, P.v, wide, P.counts, P.seen, P.mass, P.positions)


def _bad_weights(P, before, h, upto):
    """The mass of head h: NaN of the slots below `upto`, as before of the others."""
    idx = P.tables[0].long()
    mass, was = (t[idx, 0, h].reshape(-1) for t in (P.mass, before["mass"]))
    return bool(torch.isnan(mass[:upto]).all()) and torch.equal(mass[upto:], was[upto:])


@pytest.mark.parametrize("G", [1, 4, 16, 17, 40, 64])
@pytest.mark.parametrize("n,page", [(1, 16), (40, 24), (300, 16), (9001, 64)])
@pytest.mark.parametrize("room", [False, True])
def test_attention_of_logits_that_are_none(C, G, n, page, room):
    """A query that holds a NaN, and keys that all do: out, lse and the weights are NaN, not those of a query that sees nothing.
    Heads: 0 has numbers only, 1 a query with a NaN, of 2 all keys have one, of 3 a stretch of keys of the length of any part of it."""
    P = U.Paged(C, DEV, [[[n] * 4]], page=page)
    if room:
        _room_for_logits(C, P, G, 1)
    q = _queries(P, 1, 4 * G)
    q[0, 0, 0, G + G // 2, 77] = float("nan")
    at = torch.arange(n)
    at = at[(at >= n // 3) & (at < n // 3 + max(1, min(2600, n // 2)))]
    p = P.tables[0].cpu().long()[at // page]
    P.k[p.to(DEV), 0, (at % page).to(DEV), 3, 5] = float("nan")
    P.k[:, :, :, 2, 9] = float("nan")
    before = P.snapshot()
    out, lse = C.compactor_cache_attention(P.cache, q, accumulate=True, want_lse=True)
    torch.cuda.synchronize()
    bad = torch.zeros(4 * G, dtype=torch.bool, device=DEV)
    bad[G + G // 2], bad[2 * G:] = True, True
    assert torch.equal(torch.isnan(lse[0, 0, 0]), bad) and bool(torch.isfinite(lse[0, 0, 0, ~bad]).all())
    assert torch.equal(torch.isnan(out[0, 0, 0].float()), bad.view(-1, 1).expand(4 * G, 128))
    for h in (1, 2, 3):
        assert _bad_weights(P, before, h, n), h
    assert bool(torch.isfinite(P.mass[:, 0, 0]).all())


@pytest.mark.parametrize("G,T,new", [(1, 2, 2), (4, 3, 3), (4, 5, 4), (7, 6, 6), (8, 8, 8), (2, 17, 9)])
@pytest.mark.parametrize("n,page", [(20, 16), (300, 24), (9001, 64)])
@pytest.mark.parametrize("room", [False, True])
def test_attention_weights_of_none_end_where_their_query_looks(C, G, T, new, n, page, room):
    """Of several new tokens the earlier ones' queries hold a NaN: the weights of the tokens behind the last of those are numbers, the sums
    over the other queries."""
    P = U.Paged(C, DEV, [[[n]]], page=page)
    if room:
        _room_for_logits(C, P, G, T)
    q = _queries(P, T, G)
    last = (new - 1) // 2
    q[0, 0, 0, 0, 3], q[0, 0, last, G - 1, 90] = float("nan"), float("nan")
    before = P.snapshot()
    out, lse = C.compactor_cache_attention(P.cache, q, new_tokens=_new([new]), accumulate=True, want_lse=True)
    torch.cuda.synchronize()
    see = O.sees(n, new, T)
    idx = P.tables[0].long()
    mass, was = (t[idx, 0, 0].reshape(-1).double().cpu().numpy() for t in (P.mass, before["mass"]))
    assert np.isnan(mass[:see[last]]).all() and np.array_equal(mass[n:], was[n:])
    k, v, _, _, there = P.head(0, 0, 0)
    qd, od = U.f64(q), U.f64(out)
    weight, slack = np.zeros(P.capacity), np.zeros(P.capacity)
    for t in range(T):
        for g in range(G):
            if (t, g) in ((0, 0), (last, G - 1)):
                assert np.isnan(od[0, 0, t, g]).all() and bool(torch.isnan(lse[0, 0, t, g]))
                continue
            want, _, p = O.attend(qd[0, 0, t, g], k, v, see[t], there, 128 ** -0.5, 0.0)
            b_out, _, rel = U.attention_bounds(qd[0, 0, t, g], k, v, see[t], there, 128 ** -0.5, 0.0, want, p)
            assert np.all(np.abs(od[0, 0, t, g] - want) <= b_out)
            weight += p / G
            slack += p / G * (rel + 2 * U.STEP32)
    at = slice(see[last], n)
    bound = slack + (T * G + 2) * U.STEP32 * (weight + np.abs(was)) + 2.0 ** -120
    assert n > see[last] and np.all(np.abs(mass - was - weight)[at] <= bound[at])


def _weights_that_need_24_bits(n):
    """n logits x in (-1, 0), exact in bf16, whose weights w = e^x are 2^-19 or more away from the sum of two bf16 numbers.
    -> x, the two numbers, w"""
    x = -torch.arange(1, 1024, dtype=torch.float64) / 1024
    x = x[x.to(torch.bfloat16).double() == x]
    w = x.exp()
    one = w.to(torch.bfloat16).double()
    two = (w - one).to(torch.bfloat16).double()
    x, one, two, w = (t[(w - one - two).abs() >= 2.0 ** -19] for t in (x, one, two, w))
    at = torch.arange(n) % len(x)
    return x[at], one[at], two[at], w[at]


@pytest.mark.parametrize("G,T", [(1, 1), (4, 1), (4, 5), (7, 6), (8, 8)])
@pytest.mark.parametrize("page", [16, 24])
@pytest.mark.parametrize("n,tile", [(100, 0), (100, 2), (9001, 137)])
def test_attention_weights_have_all_bits(C, G, T, page, n, tile):
    """Values that cancel all but the last 8 of the 24 bits of a weight.  Row r has logits 0, 0 and x_r at three slots of one tile and
    less than -200 elsewhere, and its channel r the values -a, -b and 1 there: out = (w - a - b) / (2 + w), w = e^(x_r).
    Of |x_r| < 1 the fp32 weight is off by at most w (2^-23 for its exponential, 2 |x| 2^-24 for the argument) <= 2^-22, and the
    differences are exact in fp32; the division and the rounding to bf16 cost 2^-7 of the result at most.  A weight in 16 bits
    would give 0 in place of 2^-19 / 3 or more."""
    R = G * T
    x, a, b, w = _weights_that_need_24_bits(R)
    P = U.Paged(C, DEV, [[[n]]], page=page)
    P.k.zero_(), P.v.zero_()
    P.k[..., 127] = -200.0
    s = 32 * tile + 5
    rows = torch.arange(R)
    for slot, key, value in ((s, torch.zeros(R), -a), (s + 3, x, torch.ones(R)), (s + 17, torch.zeros(R), -b)):
        p, at = int(P.tables[0, slot // page]), slot % page
        P.k[p, 0, at, 0] = 0.0
        P.k[p, 0, at, 0, :R], P.v[p, 0, at, 0, :R] = key.to(DEV).to(torch.bfloat16), value.to(DEV).to(torch.bfloat16)
    q = torch.zeros(R, 128, dtype=torch.bfloat16, device=DEV)
    q[rows, rows], q[:, 127] = 1.0, 1.0
    out, _ = C.compactor_cache_attention(P.cache, q.view(1, 1, T, G, 128), scale=1.0, accumulate=True)
    got = out.view(R, 128).double().cpu()[rows, rows]
    want = (w - a - b) / (2 + w)
    assert bool(((got - want).abs() <= 2.0 ** -22 / (2 + w) + 2.0 ** -7 * want.abs()).all()), (got, want)


def test_attention_strides_layers_and_buffers(C):
    """q and out inside larger tensors, token-major and head-major, one layer of several, given buffers."""
    P = U.Paged(C, DEV, _counts(2, 3, 4, 70, 200, 33, 1, 150), page=16, layout="token")
    big = torch.randn(3, 2, 2, 8 + 4, 160, device=DEV).to(torch.bfloat16)          # [layer, request, token, heads, channel]
    q = big[:, :, :, 2:10, 16:144].permute(1, 0, 2, 3, 4)
    hold = torch.full((2, 2, 3, 8, 136), 9.0, device=DEV, dtype=torch.bfloat16)     # [request, token, layer, head, channel]
    out = hold[..., :128].permute(0, 2, 1, 3, 4)
    lse = torch.empty(2 * 3 * 2 * 8 + 5, device=DEV)
    got, _ = _attend_given(C, P, q, out, lse)
    assert got is out and float(hold[..., 128:].min()) == 9.0
    before = P.snapshot()
    one = P.cache.layer(1)
    o, s = C.compactor_cache_attention(one, q[:, 1:2], accumulate=True, want_lse=True)
    torch.cuda.synchronize()
    for t, l in ((0, 0), (2, 2)):
        assert torch.equal(P.mass[:, t], before["mass"][:, l])
    sub = _Sub(P, 1)
    U.check_attention(sub, q[:, 1:2], None, 128 ** -0.5, 0.0, o, s, {"mass": before["mass"][:, 1:2]}, True)


class _Sub:
    """One layer of a Paged, as the comparison sees it."""

    def __init__(self, P, l):
        self.P, self.l, self.H, self.capacity, self.dev = P, l, P.H, P.capacity, P.dev
        self.counts, self.mass = P.counts[:, l:l + 1], P.mass[:, l:l + 1]

    def head(self, b, l, h):
        return self.P.head(b, self.l, h)

    def there(self, b):
        return self.P.there(b)


def _attend_given(C, P, q, out, lse):
    before = P.snapshot()
    ws = torch.empty(C.compactor_cache_attention_workspace_size(P.cache, q, accumulate=True), dtype=torch.uint8, device=DEV)
    got, s = C.compactor_cache_attention(P.cache, q, accumulate=True, out=out, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    n = q.shape[0] * q.shape[1] * q.shape[2] * q.shape[3]
    U.check_attention(P, q, None, 128 ** -0.5, 0.0, got, s[:n].view(q.shape[:4]), before, True)
    return got, s


def test_attention_with_tables_inside_a_larger_one(C):
    P = U.Paged(C, DEV, _counts(3, 1, 2, 70, 200, 33), page=16)
    wide = torch.full((3, P.per + 9), -1, dtype=torch.int32, device=DEV)
    wide[:, 4:4 + P.per] = P.tables
    P.tables = wide[:, 4:4 + P.per]
    P.cache = P.handle()
    _attend(C, P, _queries(P, 1, 8))


def test_attention_without_state(C):
    P = U.Paged(C, DEV, _counts(2, 1, 2, 70, 200), page=16, state=False)
    _attend(C, P, _queries(P, 1, 8), accumulate=False)


def test_attention_of_more_tokens_than_promised(C):
    P = U.Paged(C, DEV, _counts(1, 1, 6, 900, 40, 100, 3000, 101, 0), page=16)
    _attend(C, P, _queries(P, 1, 24), most=100)
    _attend(C, P, _queries(P, 2, 24), most=1)
    _attend(C, P, _queries(P, 2, 24), most=10 ** 6)


@pytest.mark.parametrize("B,H,n,most", [(1, 8, 42000, 1100), (1, 1, 300000, 1100), (2, 64, 9000, 1030), (75, 8, 1500, 1100)])
def test_attention_of_many_more_tokens_than_promised(C, B, H, n, most):
    """Launches and workspace are made for `most` tokens a head; what is beyond them has to fit in."""
    P = U.Paged(C, DEV, _counts(B, 1, H, n, most, n - 77, 5), page=64)
    _attend(C, P, _queries(P, 1, 2 * H), most=most)


def test_attention_counts_outside_the_table(C):
    P = U.Paged(C, DEV, _counts(1, 1, 3, 64, 64, 64), page=16)
    P.counts[0, 0] = torch.tensor([-5, 1000, 64], dtype=torch.int32)
    out, lse = C.compactor_cache_attention(P.cache, _queries(P, 1, 6), accumulate=True, want_lse=True)
    assert not out[0, 0, 0, :2].float().any() and torch.isneginf(lse[0, 0, 0, :2]).all()
    P.counts[0, 0, 1] = 64
    want, _ = C.compactor_cache_attention(P.cache, _queries(P, 1, 6))
    assert torch.equal(U.bits(out), U.bits(want))


@pytest.mark.parametrize("counts", [[[[4000]]], [[[300, 301]], [[2, 70]]]])
def test_attention_is_the_same_twice(C, counts):
    P = U.Paged(C, DEV, counts, page=16)
    q = _queries(P, 1, 4 * P.H)
    start = P.mass.clone()
    a, la = C.compactor_cache_attention(P.cache, q, accumulate=True, want_lse=True)
    first = P.mass.clone()
    P.mass.copy_(start)
    b, lb = C.compactor_cache_attention(P.cache, q, accumulate=True, want_lse=True)
    assert torch.equal(U.bits(a), U.bits(b)) and torch.equal(la, lb) and torch.equal(first, P.mass)


def test_attention_far_into_a_large_pool(C):
    """Pages beyond 2^31 elements and 2^32 bytes."""
    page, H = 64, 8
    pages = (2 ** 31 + 2 ** 28) // (page * H * 128)
    pool = torch.empty(pages, 1, page, H, 128, dtype=torch.bfloat16, device=DEV)
    last = torch.arange(pages - 6, pages, device=DEV)
    pool[last] = torch.randn(6, 1, page, H, 128, device=DEV).to(torch.bfloat16)
    small = pool[last].clone()
    counts = torch.tensor([[[150, 384, 1, 64, 65, 300, 383, 200]]], dtype=torch.int32, device=DEV)
    q = torch.randn(1, 1, 1, 32, 128, device=DEV).to(torch.bfloat16)
    far = C.Cache(pool, pool, last.to(torch.int32).view(1, 6), counts)
    near = C.Cache(small, small, torch.arange(6, dtype=torch.int32, device=DEV).view(1, 6), counts)
    a, _ = C.compactor_cache_attention(far, q)
    b, _ = C.compactor_cache_attention(near, q)
    assert torch.equal(U.bits(a), U.bits(b)) and bool(torch.isfinite(a.float()).all())
    # and rows written there
    k = torch.randn(1, 1, 3, H, 128, device=DEV).to(torch.bfloat16)
    c2 = counts.clone()
    counts.fill_(381), c2.fill_(381)
    C.compactor_cache_append(far, k, k)
    C.compactor_cache_append(C.Cache(small, small, near.tables, c2), k, k)
    assert torch.equal(U.bits(pool[last]), U.bits(small)) and torch.equal(counts, c2) and int(counts[0, 0, 0]) == 384


def test_attention_on_another_stream(C):
    P = U.Paged(C, DEV, _counts(2, 1, 4, 2000, 700), page=16)
    q = _queries(P, 1, 16)
    want, _ = C.compactor_cache_attention(P.cache, q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        got, _ = C.compactor_cache_attention(P.cache, q, stream=side)
        torch.empty(1 << 20, device=DEV).fill_(7.0)           # would reuse scratch that was given back too early
        with torch.cuda.stream(side):
            inside, _ = C.compactor_cache_attention(P.cache, q)
    torch.cuda.synchronize()
    assert torch.equal(U.bits(got), U.bits(want)) and torch.equal(U.bits(inside), U.bits(want))


def test_a_captured_step_is_replayed_as_the_cache_grows(C):
    """Append, attention with weights, eviction in one graph, against the same calls made eagerly on a copy."""
    def make():
        P = U.Paged(C, DEV, _counts(3, 2, 4, 100, 90, 33, 140), page=16, room=80, seed=3)
        P.fill_positions()
        return P

    a, b = make(), make()
    k, v = (torch.empty(3, 2, 1, 4, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    q = torch.empty(3, 2, 1, 16, 128, dtype=torch.bfloat16, device=DEV)
    new = torch.ones(3, dtype=torch.int32, device=DEV)
    budgets = torch.tensor([120, 1000, 60], dtype=torch.int32, device=DEV)

    def step(P):
        C.compactor_cache_append(P.cache, k, v, new_tokens=new)
        out, lse = C.compactor_cache_attention(P.cache, q, new_tokens=new, accumulate=True, want_lse=True)
        C.compactor_cache_evict(P.cache, budgets=budgets, sink=2, recent=8)
        return out, lse

    for t in (k, v, q):
        t.normal_()
    warm = make()
    step(warm)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = step(a)
    g = torch.Generator(device=DEV)
    g.manual_seed(77)
    for i in range(12):
        for t in (k, v, q):
            t.copy_(torch.randn(t.shape, generator=g, device=DEV))
        new.copy_(torch.tensor([1, i % 2, 1 if i < 6 else 0], dtype=torch.int32))
        graph.replay()
        want = step(b)
        torch.cuda.synchronize()
        assert torch.equal(U.bits(got[0]), U.bits(want[0])) and torch.equal(got[1], want[1]), i
        U.same_pool(a, b.snapshot(), "replay %d" % i)


@pytest.mark.parametrize("T,scope", [(1, 0), (5, 1)])
def test_a_captured_step_over_long_heads(C, T, scope):
    """The same with heads that several workgroups share, and evictions of several launches: two graphs of one workspace each,
    replayed in turn with eager work between."""
    def make():
        P = U.Paged(C, DEV, _counts(2, 1, 4, 3000, 5000, 17, 4100, 2900), page=32, room=200, seed=6)
        P.fill_positions()
        return P

    a, b = make(), make()
    g = torch.Generator(device=DEV)
    g.manual_seed(31)
    k, v = (torch.empty(2, 1, T, 4, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    q = torch.empty(2, 1, T, 16, 128, dtype=torch.bfloat16, device=DEV)
    new = torch.tensor([T, 1], dtype=torch.int32, device=DEV)
    n = max(C.compactor_cache_attention_workspace_size(a.cache, q, accumulate=True),
            C.compactor_cache_evict_workspace_size(a.cache, scope=1))
    shared = torch.empty(n, dtype=torch.uint8, device=DEV)
    budgets = torch.tensor([2600, 2500], dtype=torch.int32, device=DEV)

    def step(P, ws):
        C.compactor_cache_append(P.cache, k, v, new_tokens=new)
        return C.compactor_cache_attention(P.cache, q, new_tokens=new, accumulate=True, want_lse=True, workspace=ws)

    def trim(P, ws):
        C.compactor_cache_evict(P.cache, budgets=budgets, sink=2, recent=8, scope=scope, workspace=ws)

    for t in (k, v, q):
        t.normal_()
    warm = make()
    step(warm, shared), trim(warm, shared)
    torch.cuda.synchronize()
    side, first, second = torch.cuda.Stream(), torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(first, stream=side):
        got = step(a, shared)
    with torch.cuda.graph(second, stream=side):
        trim(a, shared)
    for i in range(6):
        for t in (k, v, q):
            t.copy_(torch.randn(t.shape, generator=g, device=DEV))
        new.copy_(torch.tensor([T, i % 2], dtype=torch.int32))
        first.replay()
        want = step(b, None)
        torch.cuda.synchronize()
        assert torch.equal(U.bits(got[0]), U.bits(want[0])) and torch.equal(got[1], want[1]), i
        if i % 2:
            budgets.sub_(100)
            second.replay()
            trim(b, None)
        U.same_pool(a, b.snapshot(), "replay %d" % i)


@pytest.mark.parametrize("pages", [(1 << 17) - 5, 1 << 17, (1 << 17) + 1])
def test_slots_far_apart(C, pages):
    """Slot strides around the 2^24 elements up to which a lane's place in a page has 32 bits."""
    pool = [torch.empty(16, pages, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    far = [p.view(16, pages, 1, 1, 128).permute(1, 2, 0, 3, 4) for p in pool]
    at = torch.tensor([pages - 1, 3, pages // 2, 0], device=DEV)
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    near = [torch.randn(4, 1, 16, 1, 128, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2)]
    for f, n in zip(far, near):
        f[at] = n
    q = torch.randn(1, 1, 3, 4, 128, generator=g, device=DEV).to(torch.bfloat16)
    k = torch.randn(1, 1, 3, 1, 128, generator=g, device=DEV).to(torch.bfloat16)
    made = []
    for pages_of, table, n in ((far, at, pages), (near, torch.arange(4, device=DEV), 4)):
        counts, seen = (torch.full((1, 1, 1), 58, dtype=torch.int32, device=DEV) for _ in range(2))
        mass, pos = torch.zeros(n, 1, 1, 16, device=DEV), torch.zeros(n, 1, 1, 16, dtype=torch.int32, device=DEV)
        cache = C.Cache(pages_of[0], pages_of[1], table.to(torch.int32).view(1, 4), counts, seen, mass, pos)
        C.compactor_cache_append(cache, k, k)
        out, lse = C.compactor_cache_attention(cache, q, want_lse=True)
        keys, values = (U.f64(p[table].reshape(64, 128)) for p in pages_of)
        for t, see in enumerate(O.sees(61, 3, 3)):
            for h in range(4):
                args = (U.f64(q[0, 0, t, h]), keys, values, see, np.ones(64, bool), 128 ** -0.5, 0.0)
                want, want_lse, p = O.attend(*args)
                b_out, b_lse, _ = U.attention_bounds(*args, want, p)
                assert np.all(np.abs(U.f64(out[0, 0, t, h]) - want) <= b_out) and abs(float(lse[0, 0, t, h]) - want_lse) <= b_lse
        mass[table] = torch.arange(64, device=DEV, dtype=torch.float32).mul(37).remainder(64).view(4, 1, 1, 16)
        C.compactor_cache_evict(cache, budget=20)
        made.append([counts, mass[table], pos[table]] + [U.bits(p[table]) for p in pages_of])
    assert all(torch.equal(x, y) for x, y in zip(*made)) and int(made[0][0]) == 20


def test_contexts_that_share_pages(C):
    """A common prefix: pages that two contexts name, and one that names a page twice."""
    P = U.Paged(C, DEV, _counts(3, 1, 2, 150, 130, 160), page=16)
    P.tables[1, :4] = P.tables[0, :4]
    P.tables[2, 5] = P.tables[2, 2]
    _attend(C, P, _queries(P, 1, 8), accumulate=False)


@pytest.mark.parametrize("shift", [128, 64])
def test_keys_and_values_in_one_row(C, shift):
    """V beside K in a slot, and V a part of K's row."""
    P = U.Paged(C, DEV, _counts(2, 1, 2, 150, 90, 33), page=16, room=8)
    row = torch.randn(P.pages, 1, 16, 2, 128 + shift, device=DEV).to(torch.bfloat16)
    P.k, P.v = row[..., :128], row[..., shift:]
    P.fill_positions()
    P.cache = P.handle()
    _attend(C, P, _queries(P, 1, 8))
    _check_evict(C, P, [60, 50], 2, 5)
    _attend(C, P, _queries(P, 1, 8))


# ------------------------------------------------------------------------------------------ append
def _check_append(C, P, T, new=None, what="", stride=1):
    g = torch.Generator(device=DEV)
    g.manual_seed(T + 50)
    k, v = (torch.randn(P.B, P.L, T * stride, P.H, 128, generator=g, device=DEV).to(torch.bfloat16)[:, :, ::stride] for _ in range(2))
    want = P.snapshot()
    for b in range(P.B):
        n = T if new is None else min(max(int(new[b]), 0), T)
        there, t_np = P.there(b)
        for l in range(P.L):
            for h in range(P.H):
                c = min(max(int(P.counts[b, l, h]), 0), P.capacity)
                rows, c2, seen2 = O.append(c, int(P.seen[b, l, h]), n, P.capacity)
                for t, s, pos in rows:
                    if there[s]:
                        p, a = int(t_np[s // P.page]), s % P.page
                        want["k"][p, l, a, h], want["v"][p, l, a, h] = k[b, l, t, h], v[b, l, t, h]
                        if P.state:
                            want["mass"][p, l, h, a], want["positions"][p, l, h, a] = 0.0, pos
                if n > 0:
                    want["counts"][b, l, h] = c2
                    if P.state:
                        want["seen"][b, l, h] = seen2
    C.compactor_cache_append(P.cache, k, v, new_tokens=_new(new))
    torch.cuda.synchronize()
    U.same_pool(P, want, what)


@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 16, 63, 64, 65, 130])
@pytest.mark.parametrize("page,layout,state", [(16, "token", True), (7, "head", True), (64, "layer", False)])
def test_append(C, T, page, layout, state):
    P = U.Paged(C, DEV, _counts(3, 2, 3, 0, 1, 15, 16, 40), page=page, room=T, layout=layout, state=state)
    _check_append(C, P, T, what="all rows")
    P = U.Paged(C, DEV, _counts(3, 1, 3, 0, 1, 15, 16, 40), page=page, room=T, layout=layout, state=state)
    _check_append(C, P, T, new=[0, T, max(1, T // 2)], what="padded")
    P = U.Paged(C, DEV, _counts(3, 1, 3, 0, 1, 15, 16, 40), page=page, room=T, layout=layout, state=state)
    _check_append(C, P, T, new=[-4, T + 9, 1], what="counts of new tokens outside their range", stride=2)


@pytest.mark.parametrize("T", [5, 40, 200])
def test_append_beyond_the_table(C, T):
    P = U.Paged(C, DEV, _counts(2, 1, 3, 10, 32, 20, 29), page=8)
    P.tables[1, 2] = -1
    P.tables[0, 3] = 10 ** 6
    _check_append(C, P, T)


# ------------------------------------------------------------------------------------------ eviction
def _check_evict(C, P, budgets, sink=0, recent=0, scope=0, most=0, what="", given=True):
    want = P.snapshot()
    for b in range(P.B):
        there, t_np = P.there(b)
        for l in range(P.L):
            pools = [[h] for h in range(P.H)] if scope == 0 else [list(range(P.H))]
            for pool in pools:
                counts = [min(max(int(P.counts[b, l, h]), 0), P.capacity) for h in pool]
                budget = len(pool) * max(0, budgets[b])
                if sum(counts) <= budget or (most and max(counts) > most):
                    continue
                keys = []
                for h, c in zip(pool, counts):
                    _, _, mass, pos, _ = P.head(b, l, h)
                    keys.append(O.rank_keys(mass[:c], pos[:c], there[:c], int(P.seen[b, l, h]), sink, recent))
                for h, c, stay in zip(pool, counts, O.evict_keep(keys, budget)):
                    want["counts"][b, l, h] = len(stay)
                    for to, frm in O.evict_moves(stay, c):
                        if there[to] and there[frm]:
                            p, a, p2, a2 = int(t_np[to // P.page]), to % P.page, int(t_np[frm // P.page]), frm % P.page
                            want["k"][p, l, a, h], want["v"][p, l, a, h] = P.k[p2, l, a2, h], P.v[p2, l, a2, h]
                            want["mass"][p, l, h, a] = P.mass[p2, l, h, a2]
                            want["positions"][p, l, h, a] = P.positions[p2, l, h, a2]
    if given:
        C.compactor_cache_evict(P.cache, budgets=torch.tensor(budgets, dtype=torch.int32, device=DEV), sink=sink, recent=recent,
                                scope=scope, max_tokens=most)
    else:
        C.compactor_cache_evict(P.cache, budget=budgets[0], sink=sink, recent=recent, scope=scope, max_tokens=most)
    torch.cuda.synchronize()
    U.same_pool(P, want, what)


@pytest.mark.parametrize("scope", [0, 1])
@pytest.mark.parametrize("page,layout", [(16, "token"), (7, "head"), (128, "layer")])
@pytest.mark.parametrize("sink,recent", [(0, 0), (4, 16), (0, 100)])
def test_evict(C, scope, page, layout, sink, recent):
    P = U.Paged(C, DEV, _counts(3, 2, 5, 0, 1, 64, 65, 130, 257, 300), page=page, layout=layout)
    P.fill_positions()
    _check_evict(C, P, [60, 129, 1], sink, recent, scope, what="ragged budgets")
    _check_evict(C, P, [20, 20, 20], sink, recent, scope, what="again", given=False)
    _check_evict(C, P, [-7, 0, 3], sink, recent, scope, what="down to nothing")


@pytest.mark.parametrize("scope", [0, 1])
def test_evict_ties_and_numbers_that_are_none(C, scope):
    """Few different weights, zeros of both signs, infinities and NaN: the lower (head, slot) stays."""
    P = U.Paged(C, DEV, _counts(2, 1, 4, 200, 190, 50, 3, 400), page=16)
    P.fill_positions()
    v = torch.tensor([0.0, -0.0, 1.0, 1.0, float("nan"), float("inf"), -float("inf"), 1e-42, -2.0], device=DEV)
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    P.mass.copy_(v[torch.randint(0, 9, P.mass.shape, generator=g, device=DEV)])
    for budgets in ([150, 160], [100, 90], [40, 30], [9, 20], [2, 1]):
        _check_evict(C, P, budgets, 2, 5, scope, what=str(budgets))


def test_evict_all_weights_equal(C):
    P = U.Paged(C, DEV, _counts(1, 1, 2, 5000, 1200), page=16)
    P.fill_positions()
    P.mass.fill_(0.25)
    _check_evict(C, P, [1000], 0, 64)


@pytest.mark.parametrize("scope", [0, 1])
@pytest.mark.parametrize("spread", [0.0, 1e-7, 1e-4])
def test_evict_weights_that_crowd(C, scope, spread):
    """Weights within a few steps of each other beside some that are far away: the threshold lies in the crowd."""
    P = U.Paged(C, DEV, _counts(1, 2, 2, 5000, 700, 300, 9000), page=16)
    P.fill_positions()
    g = torch.Generator(device=DEV)
    g.manual_seed(8)
    P.mass.copy_(1.0 + spread * torch.rand(P.mass.shape, generator=g, device=DEV))
    far = torch.rand(P.mass.shape, generator=g, device=DEV)
    P.mass[far < 0.01] = 1e30
    P.mass[far > 0.99] = -1e-30
    for budget in (4000, 2500, 299, 20):
        _check_evict(C, P, [budget], 2, 30, scope, what=str(budget))


def test_evict_pools_of_many_heads(C):
    counts = [[[(7 * h) % 40 for h in range(300)]]]
    P = U.Paged(C, DEV, counts, page=8)
    P.fill_positions()
    _check_evict(C, P, [11], 1, 4, 1)
    _check_evict(C, P, [11], 1, 4, 0)


@pytest.mark.parametrize("scope", [0, 1])
def test_evict_protects_more_than_the_budget_of_long_heads(C, scope):
    P = U.Paged(C, DEV, _counts(1, 2, 3, 9000, 7000, 1, 9500), page=16)
    P.fill_positions()
    _check_evict(C, P, [200], 10, 30000, scope)


@pytest.mark.parametrize("H,lengths,page", [(4, (4096, 4000, 0, 2500), 64), (4, (4097, 4000, 0, 2500), 1), (256, (64, 3, 0, 40), 16),
                                            (257, (64, 3, 0, 40), 16), (70, (200, 1, 0, 130, 64), 24), (2, (8192, 8100), 32), (3, (0, 0, 5000), 8)])
def test_evict_layers_around_what_one_workgroup_takes(C, H, lengths, page):
    P = U.Paged(C, DEV, _counts(1, 2, H, *lengths), page=page)
    P.fill_positions()
    full = int(P.counts.max())
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    P.mass.copy_((torch.rand(P.mass.shape, generator=g, device=DEV) * 50).floor() / 50)        # many equal ones
    P.mass[torch.rand(P.mass.shape, generator=g, device=DEV) < 0.1] = float("nan")
    for budget in (full // 2, full // 3, full // 50, 0):
        _check_evict(C, P, [budget], 2, 9, 1, what="budget %d" % budget)


@pytest.mark.parametrize("scope", [0, 1])
def test_evict_protects_more_than_the_budget(C, scope):
    P = U.Paged(C, DEV, _counts(1, 2, 3, 90, 70, 100), page=16)
    P.fill_positions()
    _check_evict(C, P, [20], 10, 200, scope)


@pytest.mark.parametrize("scope", [0, 1])
def test_evict_pages_that_are_not_there(C, scope):
    P = U.Paged(C, DEV, _counts(2, 1, 3, 150, 100, 45), page=16)
    P.fill_positions()
    P.tables[0, 1] = -1
    P.tables[1, 0] = P.pages
    P.tables[1, 5] = 2 ** 30
    _check_evict(C, P, [130, 60], 3, 10, scope)
    _check_evict(C, P, [90, 40], 3, 10, scope)


@pytest.mark.parametrize("scope", [0, 1])
@pytest.mark.parametrize("counts,page", [([[[150, 100, 45]], [[64, 200, 0]]], 16), ([[[5000, 3000, 9000]], [[12000, 1, 700]]], 64),
                                         ([[[20000, 300, 17000]], [[40, 9000, 16384]]], 64)])
@pytest.mark.parametrize("number", [0.0, 0.3])
def test_evict_pages_that_are_not_there_beside_weights_that_are_none(C, scope, counts, page, number):
    """Tokens whose page is not there go first, then those whose weight is NaN: budgets that end among either, and behind all of both."""
    P = U.Paged(C, DEV, counts, page=page)
    P.seen.fill_(100000)
    g = torch.Generator(device=DEV)
    g.manual_seed(12)
    P.mass[torch.rand(P.mass.shape, generator=g, device=DEV) >= number] = float("nan")
    P.positions.copy_(torch.randint(0, 99000, P.positions.shape, device=DEV, dtype=torch.int32, generator=g))
    P.tables[0, ::3] = -1
    P.tables[1, 1::2] = P.pages + 3
    mean = [sum(c[0]) // 3 for c in counts]
    for part in (0.9, 0.7, 0.5, 0.3, 0.1):
        _check_evict(C, P, [max(1, int(part * m)) for m in mean], 2, 900, scope, what=str(part))


def test_evict_more_tokens_than_promised(C):
    for scope in (0, 1):
        P = U.Paged(C, DEV, _counts(2, 1, 3, 150, 100, 45, 30, 20, 10), page=16)
        P.fill_positions()
        _check_evict(C, P, [15, 15], 3, 2, scope, most=100)


@pytest.mark.parametrize("counts,budget,scope", [([[[40000, 33000, 100]]], 30000, 0), ([[[70001]]], 12345, 0),
                                                 ([[[32768, 32769, 5000]]], 20000, 1), ([[[16384, 16385], [16000, 20000]]], 16000, 0),
                                                 ([[[16384, 16000, 15, 9000]]], 8191, 0), ([[[4096, 4097, 8192, 0]], [[0, 0, 0, 12289]]], 3001, 1)])
def test_evict_long_heads(C, counts, budget, scope):
    P = U.Paged(C, DEV, counts, page=64)
    P.seen.fill_(100000)
    P.positions.copy_(torch.randint(0, 100000, P.positions.shape, device=DEV, dtype=torch.int32))
    # weights on a coarse grid too: many ties at the threshold
    P.mass.copy_((torch.rand_like(P.mass) * 4000).floor() / 4000)
    _check_evict(C, P, [budget] * P.B, 4, 700, scope)


# ------------------------------------------------------------------------------------------ admission and together
def _compressed(C, scope, L=2, H=3, lengths=(400, 90, 1), ratio=0.4, page=16, attn=True):
    g = torch.Generator(device=DEV)
    g.manual_seed(9)
    ks = [torch.randn(L, H, n, 128, generator=g, device=DEV).to(torch.bfloat16) for n in lengths]
    vs = [torch.randn(L, H, n, 128, generator=g, device=DEV).to(torch.bfloat16) for n in lengths]
    params = C.Params(L, H, sketch_dim=48, select_scope=scope)
    reqs = [C.Request(k_score=k, v_cache=v, ratio=ratio) for k, v in zip(ks, vs)]
    so, ko, kk = C.compactor_layout(params, reqs)
    scores = torch.rand(so[-1], generator=g, device=DEV)
    idx, cnt = C.compactor_select(params, reqs, scores)
    return ks, vs, params, reqs, so, ko, kk, scores, idx, cnt


@pytest.mark.parametrize("scope", [0, 1])
@pytest.mark.parametrize("seeded", [True, False])
@pytest.mark.parametrize("page,cut", [(16, 0), (7, 0), (16, 5)])
def test_admit(C, scope, seeded, page, cut):
    ks, vs, params, reqs, so, ko, kk, scores, idx, cnt = _compressed(C, scope, lengths=(400, 90, 1, 3000))
    L, H, B = 2, 3, 4
    most = max(min(r.k_score.shape[2], H * k if scope else k) for r, k in zip(reqs, kk))
    P = U.Paged(C, DEV, [[[most] * H] * L] * B, page=page, layout="token")
    if cut:            # tables without room for all
        P.tables = P.tables[:, :cut].contiguous()
        P.per, P.capacity = cut, cut * page
    P.tables[1, 1] = -1
    P.cache = P.handle()
    want = P.snapshot()
    idx = idx.clone()
    idx[3], idx[5] = -1, 10 ** 9                      # not tokens of the context: admitted without weight
    kept, c = idx.cpu().numpy(), cnt.cpu().numpy()
    sc = scores.cpu().numpy()
    for b, r in enumerate(reqs):
        n = r.k_score.shape[2]
        there, t_np = P.there(b)
        for l in range(L):
            pos = ko[b] + l * H * kk[b]
            for h in range(H):
                m = int(c[(b * L + l) * H + h])
                mine = kept[pos:pos + m]
                pos += m
                want["counts"][b, l, h], want["seen"][b, l, h] = min(m, P.capacity), n
                for s, tok in enumerate(mine[:P.capacity]):
                    if there[s]:
                        p, a = int(t_np[s // page]), s % page
                        want["positions"][p, l, h, a] = int(tok)
                        want["mass"][p, l, h, a] = float(sc[so[b] + (l * H + h) * n + tok]) if seeded and 0 <= tok < n else 0.0
    C.compactor_cache_admit(params, reqs, idx, cnt, P.cache, scores=scores if seeded else None)
    torch.cuda.synchronize()
    U.same_pool(P, want, "scope %d" % scope)


@pytest.mark.parametrize("scope", [0, 1])
def test_admit_more_requests_than_a_launch_takes(C, scope):
    lengths = tuple(40 + 7 * i for i in range(53))
    ks, vs, params, reqs, so, ko, kk, scores, idx, cnt = _compressed(C, scope, lengths=lengths)
    L, H, B = 2, 3, len(lengths)
    most = max(min(n, H * k if scope else k) for n, k in zip(lengths, kk))
    P = U.Paged(C, DEV, [[[most] * H] * L] * B, page=16)
    C.compactor_cache_admit(params, reqs, idx, cnt, P.cache, scores=scores)
    torch.cuda.synchronize()
    assert torch.equal(P.counts.reshape(-1), cnt) and torch.equal(P.seen[:, 0, 0].cpu(), torch.tensor(lengths, dtype=torch.int32))
    kept = idx.cpu().numpy()
    for b in (0, 23, 24, 25, 47, 48, 52):
        for l in range(L):
            at = ko[b] + l * H * kk[b]
            for h in range(H):
                n = int(cnt[(b * L + l) * H + h])
                _, _, mass, pos, _ = P.head(b, l, h)
                assert np.array_equal(pos[:n], kept[at:at + n])
                first = so[b] + (l * H + h) * lengths[b]
                assert np.array_equal(mass[:n], scores[first:first + lengths[b]].cpu().numpy()[kept[at:at + n]])
                at += n


@pytest.mark.parametrize("scope", [0, 1])
def test_a_program_that_serves(C, scope):
    """Compress, compact into pages, admit, then steps of append, attention and eviction, layer by layer as a model runs
    them, each checked against the oracle on what the step found."""
    L, H, G, page = 2, 3, 2, 16
    ks, vs, params, reqs, so, ko, kk, scores, idx, cnt = _compressed(C, scope, L, H)
    most = max(min(r.k_score.shape[2], H * k if scope else k) for r, k in zip(reqs, kk))
    P = U.Paged(C, DEV, [[[most] * H] * L] * 3, page=page, room=40)
    P.counts.zero_()
    C.compactor_compact_paged(params, reqs, idx, cnt, P.k, P.v, list(P.tables))
    C.compactor_cache_admit(params, reqs, idx, cnt, P.cache, scores=scores)
    torch.cuda.synchronize()
    # what lies in the pages are the retained rows
    pos0 = ko[0]
    c0 = int(cnt[0])
    k0 = P.k[P.tables[0].long(), 0, :, 0].reshape(-1, 128)[:c0]
    assert torch.equal(U.bits(k0), U.bits(ks[0][0, 0][idx[pos0:pos0 + c0].long()]))
    layers = [P.cache.layer(l) for l in range(L)]
    g = torch.Generator(device=DEV)
    g.manual_seed(21)
    budgets = [max(4, k) for k in kk]
    for step, T in enumerate([1, 1, 4, 1, 3, 1]):
        k, v = (torch.randn(3, L, T, H, 128, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
        q = torch.randn(3, L, T, H * G, 128, generator=g, device=DEV).to(torch.bfloat16)
        new = [T, max(0, T - 1), T]
        for l in range(L):
            C.compactor_cache_append(layers[l], k[:, l:l + 1], v[:, l:l + 1], new_tokens=_new(new))
            before = P.mass.clone()
            out, lse = C.compactor_cache_attention(layers[l], q[:, l:l + 1], new_tokens=_new(new), accumulate=True, want_lse=True)
            torch.cuda.synchronize()
            U.check_attention(_Sub(P, l), q[:, l:l + 1], new, 128 ** -0.5, 0.0, out, lse, {"mass": before[:, l:l + 1]}, True,
                              what="step %d layer %d" % (step, l))
        if step % 2:
            _check_evict(C, P, budgets, 1, 3, scope, what="step %d" % step)
    assert int(P.seen[0, 0, 0]) == 400 + 11
