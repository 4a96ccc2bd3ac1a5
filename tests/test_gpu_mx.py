"""The paged cache in 4 bits against the float64 oracles: rows in and out, attention, eviction, alone and together."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as O
from oracle import mx_oracle as M
from tests import cache_util as U
from tests import gpu_util as GU
from tests import mx_util as X
from tests.test_gpu_cache import DEV, _counts, _new, _queries, _Sub

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def C():
    return GU.binding()


def _rows(shape, seed=0):
    """Rows with outliers, groups of zeros, of one number, of tiny and large ones, and some that are none."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    t = torch.randn(shape, generator=g, device=DEV) * torch.exp2(torch.randint(-20, 20, (*shape[:-1], 1), generator=g, device=DEV).float())
    t[..., 7] *= 20
    flat = t.view(-1, 4, 32)
    for at, x in enumerate((0.0, -0.0, 1.0, -1.75, 3e38, -3.3895313892515355e38, 1e-38, 2.0 ** -133, float("nan"), float("inf"), -float("inf"))):
        flat[at::29, at % 4, 5 if at > 7 else slice(None)] = x
    return t.to(torch.bfloat16)


def _values(t):
    return M.decode(*M.encode(U.f64(t)))


def _same_values(got, want):
    return np.array_equal(U.f64(got), want, equal_nan=True)


# ------------------------------------------------------------------------------------------ rows
def test_every_number_of_16_bits(C):
    """Each of them as the largest of its group, and each beside larger ones: as the oracle has them, bit by bit."""
    every = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    numbers = every[torch.isfinite(every.float())]
    rows = numbers[torch.argsort(numbers.float().abs())].view(-1, 128)          # groups of nearly one size
    alone = torch.zeros(len(every), 128, dtype=torch.bfloat16)
    alone[:, 0], alone[:, 33] = every, every
    alone[:, 34] = every.roll(3000)
    rows = torch.cat((rows, alone))
    n = len(rows)
    P = X.Paged(C, DEV, [[[0]]], page=64, room=n)
    k = rows.to(DEV).view(1, 1, n, 1, 128)
    C.compactor_mx_append(P.mx, k, k.flip(2).contiguous())
    k4, v4 = C.compactor_mx_read(P.mx, n)
    codes, scales = M.encode(U.f64(rows))
    at = P.tables[0].long()
    assert np.array_equal(P.k_scales[at, 0, 0].reshape(-1, 4)[:n].cpu().numpy(), scales)
    assert np.array_equal(P.k4[at, 0, :, 0].reshape(-1, 64)[:n].cpu().numpy(), X.pack(codes))
    assert _same_values(k4.view(n, 128), M.decode(codes, scales)) and _same_values(v4.view(n, 128), M.decode(codes, scales)[::-1])


def test_every_row_of_4_bits_comes_back(C):
    """All codes beside all scales, those that no call writes among them (2^-127 to 2^127; 6 times 2^126 is an infinity in 16 bits)."""
    P = X.Paged(C, DEV, [[[256 * 8]]], page=64)
    codes = np.tile(np.arange(256, dtype=np.uint8), 256 * 8 * 64 // 256).reshape(256 * 8, 64)
    scales = np.repeat(np.arange(256, dtype=np.uint8), 32).reshape(256 * 8, 4)
    at = P.tables[0].long()
    for rows, s in ((P.k4, P.k_scales), (P.v4, P.v_scales)):
        rows[at, 0, :, 0] = torch.from_numpy(codes).to(DEV).view(-1, 64, 64)
        s[at, 0, 0] = torch.from_numpy(scales).to(DEV).view(-1, 64, 4)
    k, v = C.compactor_mx_read(P.mx, 256 * 8, first=0)
    want = torch.from_numpy(M.decode(X.unpack(codes), scales)).to(torch.bfloat16)
    for t in (k, v):
        assert np.array_equal(t.view(-1, 128).float().cpu().numpy(), want.float().numpy(), equal_nan=True)


@pytest.mark.parametrize("T,new", [(1, None), (3, [3, 0, 2]), (8, [8, 1, 9]), (9, None), (64, [64, -1, 5]), (65, [0, 65, 64]), (200, [200, 3, 130])])
@pytest.mark.parametrize("page,layout,state", [(16, "token", True), (7, "head", True), (24, "layer", False), (1, "head", True)])
def test_append_and_read(C, T, new, page, layout, state):
    counts = _counts(3, 2, 3, 40, 0, 17, 33, 100)
    P = X.Paged(C, DEV, counts, page=page, layout=layout, room=150, state=state)
    P.tables[1, (40 + T // 2) // page] = -1
    P.mx = P.mx_handle()
    want = P.snapshot()
    k, v = _rows((3, 2, T, 3, 128), T), _rows((3, 2, T, 3, 128), T + 1)
    values = [_values(t) for t in (k, v)]
    (kc, ks), (vc, vs) = (M.encode(U.f64(t)) for t in (k, v))
    read = np.zeros((2, *k.shape))
    for b in range(3):
        n = T if new is None else min(max(new[b], 0), T)
        there, t_np = P.there(b)
        for l in range(2):
            for h in range(3):
                rows, c, seen = O.append(counts[b][l][h], int(P.seen[b, l, h]), n, P.capacity)
                want["counts"][b, l, h] = c
                if state:
                    want["seen"][b, l, h] = seen
                for t, s, pos in rows:
                    if not there[s]:
                        continue
                    p, a = int(t_np[s // page]), s % page
                    for name, x, y in (("k4", kc, ks), ("v4", vc, vs)):
                        want[name][p, l, a, h] = torch.from_numpy(X.pack(x[b, l, t, h])).to(DEV)
                        want[name[0] + "_scales"][p, l, h, a] = torch.from_numpy(y[b, l, t, h].astype(np.uint8)).to(DEV)
                    if state:
                        want["mass"][p, l, h, a], want["positions"][p, l, h, a] = 0.0, pos
                # the last n slots that the head has
                for t in range(n):
                    s = c - n + t
                    if s < 0 or not there[s]:
                        continue
                    was = s - counts[b][l][h]
                    if was >= 0:
                        read[0, b, l, t, h], read[1, b, l, t, h] = values[0][b, l, was, h], values[1][b, l, was, h]
                    else:
                        p, a = int(t_np[s // page]), s % page
                        read[0, b, l, t, h], read[1, b, l, t, h] = U.f64(P.k[p, l, a, h]), U.f64(P.v[p, l, a, h])
    C.compactor_mx_append(P.mx, k, v, new_tokens=_new(new))
    X.same(P, want)
    got = C.compactor_mx_read(P.mx, T, new_tokens=_new(new))
    for t, w in zip(got, read):
        assert _same_values(t, w)


def test_read_into_larger_tensors(C):
    P = X.Paged(C, DEV, _counts(2, 2, 3, 40, 0, 17, 33, 100), page=24)
    want = C.compactor_mx_read(P.mx, 70, first=20)
    hold = torch.full((2, 2, 70, 2, 3, 136), 9.0, dtype=torch.bfloat16, device=DEV)          # [which, request, token, layer, head, channel]
    k, v = (hold[i][..., :128].permute(0, 2, 1, 3, 4) for i in range(2))
    C.compactor_mx_read(P.mx, 70, first=20, k=k, v=v)
    assert torch.equal(k, want[0]) and torch.equal(v, want[1]) and float(hold[..., 128:].min()) == 9.0
    b, l, h = 1, 1, 0
    n = int(P.counts[b, l, h])
    rows = P.head(b, l, h)[0]
    assert np.array_equal(U.f64(want[0][b, l, :max(0, n - 20), h]), rows[20:n][:70]) and not want[0][b, l, max(0, n - 20):, h].any()
    one = P.mx.layer(1)
    assert torch.equal(C.compactor_mx_read(one, 70, first=20)[0], want[0][:, 1:])


@pytest.mark.parametrize("page,to_page,layout", [(16, 16, "token"), (24, 7, "head"), (64, 16, "layer")])
@pytest.mark.parametrize("state", [True, False])
def test_store(C, page, to_page, layout, state):
    counts = _counts(3, 2, 3, 40, 0, 17, 133, 300, 64)
    S = U.Paged(C, DEV, counts, page=page, layout=layout, state=True, seed=4)
    S.fill_positions()
    S.k.copy_(_rows(S.k.shape, 5)), S.v.copy_(_rows(S.v.shape, 6))
    S.tables[1, 1] = -1
    P = X.Paged(C, DEV, _counts(3, 2, 3, 5, 250), page=to_page, state=state)
    P.tables[0, 2] = P.pages
    P.mx = P.mx_handle()
    want = P.snapshot()
    for b in range(3):
        from_there, to_there = S.there(b), P.there(b)
        for l in range(2):
            for h in range(3):
                k, v, mass, pos, _ = S.head(b, l, h)
                n = want["counts"][b, l, h] = min(counts[b][l][h], P.capacity)
                if state:
                    want["seen"][b, l, h] = S.seen[b, l, h]
                (kc, ks), (vc, vs) = (M.encode(t[:max(1, n)]) for t in (k, v))
                for s in range(n):
                    if not (from_there[0][s] and to_there[0][s]):
                        continue
                    p, a = int(to_there[1][s // to_page]), s % to_page
                    for name, x, y in (("k4", kc, ks), ("v4", vc, vs)):
                        want[name][p, l, a, h] = torch.from_numpy(X.pack(x[s])).to(DEV)
                        want[name[0] + "_scales"][p, l, h, a] = torch.from_numpy(y[s].astype(np.uint8)).to(DEV)
                    if state:
                        want["mass"][p, l, h, a], want["positions"][p, l, h, a] = float(mass[s]), int(pos[s])
    C.compactor_mx_store(P.mx, S.cache)
    X.same(P, want)


# ------------------------------------------------------------------------------------------ attention
def _attend(C, P, q, new=None, scale=0.0, cap=0.0, accumulate=True, most=0, what="", **kw):
    before = P.snapshot()
    out, lse = C.compactor_mx_attention(P.mx, q, new_tokens=_new(new), scale=scale, softcap=cap, accumulate=accumulate,
                                        max_tokens=most, want_lse=True, **kw)
    torch.cuda.synchronize()
    X.same(P, before if not accumulate else {**before, "mass": P.mass}, what=what)
    U.check_attention(P, q, new, scale or 128 ** -0.5, cap, out, lse, before, accumulate, most, what)
    return out, lse


@pytest.mark.parametrize("page,layout", [(16, "token"), (32, "head"), (64, "layer"), (7, "token"), (24, "head"), (1, "token"), (1000, "head")])
@pytest.mark.parametrize("G", [1, 4])
def test_attention_lengths(C, page, layout, G):
    counts = _counts(3, 1, 8, 0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 511, 513, 700, 1023, 1025)
    P = X.Paged(C, DEV, counts, page=page, layout=layout, gain=8.0)
    _attend(C, P, _queries(P, 1, 8 * G), what="page %d" % page)


@pytest.mark.parametrize("G,T", [(1, 1), (3, 1), (7, 1), (8, 1), (16, 1), (17, 1), (32, 1), (64, 1), (33, 1),
                                 (1, 2), (4, 5), (8, 8), (5, 3), (1, 64), (2, 17), (3, 21)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_attention_rows(C, G, T, accumulate):
    counts = _counts(2, 2, 2, 333, 80, 64, 1, 0, 40, 129, 500)
    P = X.Paged(C, DEV, counts, page=16 if T % 2 else 24, layout="token", seed=G * 100 + T)
    _attend(C, P, _queries(P, T, 2 * G), accumulate=accumulate, what="G %d T %d" % (G, T))
    new = [T // 2, T + 5] if T > 1 else [0, 1]
    _attend(C, P, _queries(P, T, 2 * G), new=new, accumulate=accumulate, what="G %d T %d, padded" % (G, T))
    _attend(C, P, _queries(P, T, 2 * G), new=[-3, 1], accumulate=accumulate, what="G %d T %d, one token" % (G, T))


@pytest.mark.parametrize("scale,cap,gain", [(0.0, 30.0, 1.0), (0.5, 5.0, 8.0), (0.02, 0.0, 8.0), (1.0, 0.0, 20.0), (1.0, 50.0, 20.0), (0.0, 1e4, 1.0)])
def test_attention_scales_and_caps(C, scale, cap, gain):
    P = X.Paged(C, DEV, _counts(2, 1, 4, 700, 33, 5, 1500), page=16, gain=gain)
    _attend(C, P, _queries(P, 2, 16), scale=scale, cap=cap)


@pytest.mark.parametrize("B,L,H,n,page", [(1, 1, 4, 9001, 64), (2, 1, 1, 33000, 24), (1, 3, 2, 6007, 32), (1, 1, 2, 70001, 256)])
@pytest.mark.parametrize("G,T", [(4, 1), (7, 1), (5, 4)])
def test_attention_long(C, B, L, H, n, page, G, T):
    P = X.Paged(C, DEV, _counts(B, L, H, n, n - 3 * page - 1, 5), page=page, layout="head")
    _attend(C, P, _queries(P, T, H * G), cap=20.0 if T > 1 else 0.0)


@pytest.mark.parametrize("B,L,H,n,page,G,T", [(43, 1, 5, 1500, 16, 5, 1), (37, 1, 3, 1400, 24, 3, 5), (41, 3, 3, 3000, 16, 3, 1)])
def test_attention_of_many_rows_in_fragments(C, B, L, H, n, page, G, T):
    """Numbers of rows that are no multiple of four."""
    P = X.Paged(C, DEV, _counts(B, L, H, n, n - 3 * page - 1, 5), page=page, layout="token")
    _attend(C, P, _queries(P, T, H * G))


@pytest.mark.parametrize("H,lengths,page", [(2, (9001, 300, 0, 1), 64), (1, (20011, 6000, 4500, 31), 24)])
@pytest.mark.parametrize("G,T", [(8, 5), (64, 1), (1, 33), (4, 5)])
@pytest.mark.parametrize("room", [0, 2 ** 28 + 1])
def test_attention_weights_of_many_rows(C, H, lengths, page, G, T, room):
    P = X.Paged(C, DEV, _counts(4, 1, H, *lengths), page=page)
    P.tables[1, 1] = -1
    P.mx = P.mx_handle()
    if room:
        wide = torch.full((4, room // (4 * H * G * T * page * 4) + 1), -1, dtype=torch.int32, device=DEV)
        wide[:, :P.per] = P.tables
        P.mx = C.MxCache(P.k4, P.v4, P.k_scales, P.v_scales, wide, P.counts, P.seen, P.mass, P.positions)
    cap = 15.0 if T == 5 else 0.0
    _attend(C, P, _queries(P, T, H * G), cap=cap)
    _attend(C, P, _queries(P, T, H * G), new=[T - 1, 0, T, 1], cap=cap, most=9000 if H == 2 else 0)


@pytest.mark.parametrize("page", [16, 24])
@pytest.mark.parametrize("T", [1, 9])
def test_attention_of_one_long_request_among_many(C, page, T):
    """A wave has more tiles than it keeps places for."""
    P = X.Paged(C, DEV, [[[34001, 40, 0, 20000, 33999, 1, 128, 16385]]], page=page)
    B = 66
    tables = torch.full((B, P.per), -1, dtype=torch.int32, device=DEV)
    tables[0] = P.tables[0]
    counts, seen = (torch.zeros(B, 1, 8, dtype=torch.int32, device=DEV) for _ in range(2))
    counts[0] = P.counts[0]
    cache = C.MxCache(P.k4, P.v4, P.k_scales, P.v_scales, tables, counts, seen, P.mass, P.positions)
    q = torch.zeros(B, 1, T, 32, 128, dtype=torch.bfloat16, device=DEV)
    q[:1] = _queries(P, T, 32)
    before = P.snapshot()
    out, lse = C.compactor_mx_attention(cache, q, accumulate=True, want_lse=True)
    torch.cuda.synchronize()
    assert not out[1:].float().any() and torch.isneginf(lse[1:]).all()
    U.check_attention(P, q[:1], None, 128 ** -0.5, 0.0, out[:1], lse[:1], before, True)


@pytest.mark.parametrize("B,L,H,lengths", [(5, 2, 9, (2000, 1, 0, 1025, 700, 128, 129, 1999)), (43, 1, 7, (1100, 30, 0, 1500)),
                                           (65, 1, 8, (1100, 5, 900, 0, 1400)), (200, 3, 7, (40, 1100, 0))])
def test_attention_of_many_heads(C, B, L, H, lengths):
    P = X.Paged(C, DEV, _counts(B, L, H, *lengths), page=32, layout="token", seed=B)
    _attend(C, P, _queries(P, 2, H), new=None if B % 2 else [b % 3 for b in range(B)], what="%d heads" % (B * L * H))


@pytest.mark.parametrize("page", [16, 24, 128])
def test_attention_does_not_look_past_the_end(C, page):
    """Slots that no token is in, pages that nobody names, and pages that are not there hold NaN."""
    P = X.Paged(C, DEV, _counts(2, 1, 4, 0, 1, 45, 100, 300, 31, 33, 250), page=page, room=60, fill=255)
    P.tables[1, 1] = -1
    P.tables[0, 0] = P.pages + 7
    P.mx = P.mx_handle()
    _attend(C, P, _queries(P, 3, 12))
    _attend(C, P, _queries(P, 3, 12), new=[2, 1], accumulate=False)
    _attend(C, P, _queries(P, 8, 32), new=[7, 8])


@pytest.mark.parametrize("count,T,G", [(40, 4, 2), (33, 2, 8), (64, 5, 4), (3, 5, 1), (130, 7, 2), (18, 16, 2), (2000, 3, 20)])
@pytest.mark.parametrize("page", [16, 24])
def test_attention_does_not_look_ahead(C, count, T, G, page):
    """A later token's row with a group that is NaN: the queries that see it have NaN in that group's channels and numbers in the others."""
    P = X.Paged(C, DEV, [[[count, count]]], page=page)
    q = _queries(P, T, 2 * G)
    clean, _ = C.compactor_mx_attention(P.mx, q)
    first = T - 1 if T < 3 else T - 2                    # the first query that sees slot s
    s = count - T + first
    for h in range(2):
        P.v_scales[int(P.tables[0, s // page]), 0, h, s % page, 1 + h] = 255
    P.k_scales[int(P.tables[0, s // page]), 0, 1, s % page, 3] = 255
    out, lse = C.compactor_mx_attention(P.mx, q, want_lse=True)
    torch.cuda.synchronize()
    for t, see in enumerate(O.sees(count, T, T)):
        for h in range(2):
            rows = out[0, 0, t, h * G:(h + 1) * G].float()
            if see <= s:
                assert torch.equal(rows, clean[0, 0, t, h * G:(h + 1) * G].float()), (t, h)
            elif h == 0:
                assert torch.isnan(rows[:, 32:64]).all()
                rest = torch.cat((rows[:, :32], rows[:, 64:]), 1)
                assert torch.equal(rest, torch.cat((clean[0, 0, t, :G, :32], clean[0, 0, t, :G, 64:]), 1).float())
            else:
                assert torch.isnan(rows).all() and torch.isnan(lse[0, 0, t, G:]).all()


@pytest.mark.parametrize("n,page", [(1, 16), (40, 24), (9001, 64)])
@pytest.mark.parametrize("G", [1, 17, 64])
def test_attention_of_logits_that_are_none(C, G, n, page):
    P = X.Paged(C, DEV, [[[n] * 2]], page=page)
    q = _queries(P, 1, 2 * G)
    q[0, 0, 0, G // 2, 77] = float("nan")
    before = P.snapshot()
    out, lse = C.compactor_mx_attention(P.mx, q, accumulate=True, want_lse=True)
    torch.cuda.synchronize()
    bad = torch.zeros(2 * G, dtype=torch.bool, device=DEV)
    bad[G // 2] = True
    assert torch.equal(torch.isnan(lse[0, 0, 0]), bad) and torch.equal(torch.isnan(out[0, 0, 0].float()), bad.view(-1, 1).expand(2 * G, 128))
    idx = P.tables[0].long()
    mass, was = (t[idx, 0, 0].reshape(-1) for t in (P.mass, before["mass"]))
    assert bool(torch.isnan(mass[:n]).all()) and torch.equal(mass[n:], was[n:]) and bool(torch.isfinite(P.mass[:, 0, 1]).all())


def test_attention_strides_layers_and_buffers(C):
    P = X.Paged(C, DEV, _counts(2, 3, 4, 70, 200, 33, 1, 150), page=16, layout="token")
    big = torch.randn(3, 2, 2, 8 + 4, 160, device=DEV).to(torch.bfloat16)          # [layer, request, token, heads, channel]
    q = big[:, :, :, 2:10, 16:144].permute(1, 0, 2, 3, 4)
    hold = torch.full((2, 2, 3, 8, 136), 9.0, device=DEV, dtype=torch.bfloat16)     # [request, token, layer, head, channel]
    out, lse = hold[..., :128].permute(0, 2, 1, 3, 4), torch.empty(2, 3, 2, 8, device=DEV)
    ws = torch.empty(C.compactor_mx_attention_workspace_size(P.mx, q, accumulate=True), dtype=torch.uint8, device=DEV)
    before = P.snapshot()
    got, _ = C.compactor_mx_attention(P.mx, q, accumulate=True, out=out, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    assert got is out and float(hold[..., 128:].min()) == 9.0
    U.check_attention(P, q, None, 128 ** -0.5, 0.0, out, lse, before, True)
    before = P.snapshot()
    o, s = C.compactor_mx_attention(P.mx.layer(1), q[:, 1:2], accumulate=True, want_lse=True)
    torch.cuda.synchronize()
    assert torch.equal(P.mass[:, ::2], before["mass"][:, ::2])
    U.check_attention(_Sub(P, 1), q[:, 1:2], None, 128 ** -0.5, 0.0, o, s, {"mass": before["mass"][:, 1:2]}, True)


def test_attention_without_state_and_of_more_tokens_than_promised(C):
    P = X.Paged(C, DEV, _counts(2, 1, 2, 70, 200), page=16, state=False)
    _attend(C, P, _queries(P, 1, 8), accumulate=False)
    P = X.Paged(C, DEV, _counts(1, 1, 6, 900, 40, 100, 3000, 101, 0), page=16)
    _attend(C, P, _queries(P, 1, 24), most=100)
    P.counts[0, 0, :2] = torch.tensor([-5, 100000], dtype=torch.int32)
    _attend(C, P, _queries(P, 2, 24), most=1)


def test_far_into_a_large_pool(C):
    """Pages beyond 2^32 bytes."""
    page, H = 64, 8
    pages = (2 ** 32 + 2 ** 28) // (page * H * 64)
    pool = torch.empty(pages, 1, page, H, 64, dtype=torch.uint8, device=DEV)
    scales = torch.empty(pages, 1, H, page, 4, dtype=torch.uint8, device=DEV)
    last = torch.arange(pages - 6, pages, device=DEV)
    pool[last] = torch.randint(0, 256, (6, 1, page, H, 64), device=DEV, dtype=torch.uint8)
    scales[last] = torch.randint(120, 132, (6, 1, H, page, 4), device=DEV, dtype=torch.uint8)
    small, small_scales = pool[last].clone(), scales[last].clone()
    counts = torch.tensor([[[150, 384, 1, 64, 65, 300, 383, 200]]], dtype=torch.int32, device=DEV)
    q = torch.randn(1, 1, 1, 32, 128, device=DEV).to(torch.bfloat16)
    far = C.MxCache(pool, pool, scales, scales, last.to(torch.int32).view(1, 6), counts)
    near = C.MxCache(small, small, small_scales, small_scales, torch.arange(6, dtype=torch.int32, device=DEV).view(1, 6), counts.clone())
    a, b = (C.compactor_mx_attention(c, q)[0] for c in (far, near))
    assert torch.equal(U.bits(a), U.bits(b)) and bool(torch.isfinite(a.float()).all())
    far.counts.fill_(381), near.counts.fill_(381)
    k = torch.randn(1, 1, 3, H, 128, device=DEV).to(torch.bfloat16)
    for c in (far, near):
        C.compactor_mx_append(c, k, k)
    assert torch.equal(pool[last], small) and torch.equal(scales[last], small_scales)
    assert torch.equal(C.compactor_mx_read(far, 3)[0], C.compactor_mx_read(near, 3)[0])


# ------------------------------------------------------------------------------------------ eviction, and together
@pytest.mark.parametrize("scope", [0, 1])
@pytest.mark.parametrize("counts,page", [([[[150, 100, 45]], [[64, 200, 0]]], 16), ([[[5000, 3000, 9000]], [[20000, 1, 700]]], 24)])
def test_evict(C, scope, counts, page):
    """The slots that a cache of 16 bits with the same state keeps, where it moves them."""
    P = X.Paged(C, DEV, counts, page=page, layout="head")
    P.seen.fill_(30000)
    P.positions.copy_(torch.randint(0, 30000, P.positions.shape, device=DEV, dtype=torch.int32))
    P.tables[0, 1] = -1
    for share in (2, 3, 20):
        twin = [t.clone() for t in (P.counts, P.seen, P.mass, P.positions)]
        other = C.Cache(P.k, P.v, P.tables, *twin)          # holds the same values, and moves them
        budget = max(int(P.counts.max()) // share, 3)
        C.compactor_cache_evict(other, budget=budget, sink=2, recent=40, scope=scope)
        C.compactor_mx_evict(P.mx, budget=budget, sink=2, recent=40, scope=scope)
        for t, w in zip((P.counts, P.seen, P.positions, P.mass), (twin[0], twin[1], twin[3], twin[2])):
            assert torch.equal(t, w)
        moved = P.k.clone(), P.v.clone()
        P.values()
        for t, w in zip((P.k, P.v), moved):
            assert torch.equal(U.bits(t), U.bits(w))


def test_on_another_stream(C):
    P = X.Paged(C, DEV, _counts(2, 1, 4, 2000, 700), page=16)
    q = _queries(P, 1, 16)
    want, _ = C.compactor_mx_attention(P.mx, q)
    rows = C.compactor_mx_read(P.mx, 300, first=1500)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        got, _ = C.compactor_mx_attention(P.mx, q, stream=side)
        read = C.compactor_mx_read(P.mx, 300, first=1500, stream=side)
        torch.empty(1 << 20, device=DEV).fill_(7.0)
    torch.cuda.synchronize()
    assert torch.equal(U.bits(got), U.bits(want)) and torch.equal(read[0], rows[0]) and torch.equal(read[1], rows[1])


@pytest.mark.parametrize("T,counts", [(1, (100, 90, 33, 140)), (5, (3000, 5000, 17, 4100))])
def test_a_captured_step_is_replayed_as_the_cache_grows(C, T, counts):
    """Append, attention with weights, eviction in one graph, against the same calls made eagerly on a copy."""
    def make():
        P = X.Paged(C, DEV, _counts(3, 1, 4, *counts), page=16, room=80, seed=3)
        P.fill_positions()
        return P

    a, b = make(), make()
    k, v = (torch.empty(3, 1, T, 4, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    q = torch.empty(3, 1, T, 16, 128, dtype=torch.bfloat16, device=DEV)
    new = torch.ones(3, dtype=torch.int32, device=DEV)
    budgets = torch.tensor([120, 100000, 60], dtype=torch.int32, device=DEV)

    def step(P):
        C.compactor_mx_append(P.mx, k, v, new_tokens=new)
        out, lse = C.compactor_mx_attention(P.mx, q, new_tokens=new, accumulate=True, want_lse=True)
        C.compactor_mx_evict(P.mx, budgets=budgets, sink=2, recent=8)
        return out, lse, *C.compactor_mx_read(P.mx, T, new_tokens=new)

    for t in (k, v, q):
        t.normal_()
    step(make())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        got = step(a)
    g = torch.Generator(device=DEV)
    g.manual_seed(77)
    for i in range(8):
        for t in (k, v, q):
            t.copy_(torch.randn(t.shape, generator=g, device=DEV))
        new.copy_(torch.tensor([T, i % 2, T if i < 6 else 0], dtype=torch.int32))
        graph.replay()
        want = step(b)
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x, y), i
        X.same(a, b.snapshot(), what="replay %d" % i)


def test_a_program_that_serves(C):
    """A cache of 16 bits becomes one of 4, then steps of append, attention and eviction, layer by layer, each checked against the oracle."""
    L, H, G, page = 2, 3, 2, 16
    S = U.Paged(C, DEV, _counts(3, L, H, 160, 36, 1, 90), page=page, seed=8)
    S.fill_positions()
    P = X.Paged(C, DEV, _counts(3, L, H, 160), page=24, room=40)
    C.compactor_mx_store(P.mx, S.cache)
    assert torch.equal(P.counts, S.counts) and torch.equal(P.seen, S.seen)
    layers = [P.mx.layer(l) for l in range(L)]
    g = torch.Generator(device=DEV)
    g.manual_seed(21)
    for step, T in enumerate([1, 1, 4, 1, 3]):
        k, v = (torch.randn(3, L, T, H, 128, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
        q = torch.randn(3, L, T, H * G, 128, generator=g, device=DEV).to(torch.bfloat16)
        new = [T, max(0, T - 1), T]
        for l in range(L):
            C.compactor_mx_append(layers[l], k[:, l:l + 1], v[:, l:l + 1], new_tokens=_new(new))
            P.values()
            before = P.mass.clone()
            out, lse = C.compactor_mx_attention(layers[l], q[:, l:l + 1], new_tokens=_new(new), accumulate=True, want_lse=True)
            torch.cuda.synchronize()
            U.check_attention(_Sub(P, l), q[:, l:l + 1], new, 128 ** -0.5, 0.0, out, lse, {"mass": before[:, l:l + 1]}, True,
                              what="step %d layer %d" % (step, l))
        if step % 2:
            C.compactor_mx_evict(P.mx, budget=80, sink=1, recent=3)
            assert int(P.counts.max()) <= 80
    assert torch.equal(P.seen[0], S.seen[0] + 10)
