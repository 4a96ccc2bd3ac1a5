"""The pages of caches against the plain oracle, and rows and state after their copies."""
import numpy as np
import pytest
import torch

from oracle import pages_oracle as O
from tests import cache_util as U
from tests import gpu_util as GU
from tests import mx_util as X
from tests.test_gpu_cache import DEV, _counts, _new, _queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def C():
    return GU.binding()


class World:
    """A pool whose pages requests share: tables, counts and refs on the GPU, and what the oracle makes of them."""

    def __init__(self, C, counts, page=16, entries=None, spare=20, mx=False, layout="token", seed=1, state=True, foreign=2):
        self.C, self.mx, rng = C, mx, np.random.default_rng(seed)
        make = X.Paged if mx else U.Paged
        self.P = P = make(C, DEV, counts, page=page, layout=layout, seed=seed, spare=spare, state=state)
        self.page, self.entries = page, entries or P.per
        self.counts = [[n for l in b for n in l] for b in counts]
        order = list(rng.permutation(P.pages))
        self.refs = [0] * P.pages
        for _ in range(foreign):                    # somebody else's
            self.refs[order.pop()] = 1
        self.tables = []
        for b in self.counts:
            n = min(-(-max(b) // page), self.entries)
            self.tables.append([int(order.pop()) for _ in range(n)] + [-1] * (self.entries - n))
            for p in self.tables[-1][:n]:
                self.refs[p] += 1

    def share(self, groups):
        """groups: (from, to, entries): `to` has the first entries of `from`."""
        for a, b, n in groups:
            for i in range(n):
                old, new = self.tables[b][i], self.tables[a][i]
                if 0 <= old < len(self.refs):
                    self.refs[old] -= 1
                if 0 <= new < len(self.refs):
                    self.refs[new] += 1
                self.tables[b][i] = new

    def load(self):
        P = self.P
        P.tables = torch.tensor(self.tables, dtype=torch.int32, device=DEV)
        P.per, P.capacity = self.entries, self.entries * self.page
        P.counts.copy_(torch.tensor(self.counts, dtype=torch.int32).view(P.counts.shape))
        self.dev_refs = torch.tensor(self.refs, dtype=torch.int32, device=DEV)
        self.seen = P.seen.cpu().view(P.B, -1).tolist()
        self.cache = P.mx_handle() if self.mx else P.handle()
        self.held = [[min(max(n, 0), P.capacity) for n in b] for b in self.counts]
        self.rows = {n: getattr(P, n).clone() for n in (X.ROWS if self.mx else ("k", "v")) + ("mass", "positions")}

    def copy(self, pairs, done, want):
        (self.C.compactor_mx_pages_copy if self.mx else self.C.compactor_pages_copy)(self.cache, pairs, done)
        torch.cuda.synchronize()
        for n, t in self.rows.items():
            if n in ("mass", "positions") and not self.P.state:
                continue
            for a, b in want:
                t[b] = t[a]
            got = getattr(self.P, n)
            assert torch.equal(got if got.dtype != torch.bfloat16 else U.bits(got), t if t.dtype != torch.bfloat16 else U.bits(t)), n

    def same(self, what=""):
        assert self.P.tables.tolist() == self.tables, what + ": tables"
        assert self.dev_refs.tolist() == self.refs, what + ": refs"
        assert self.P.counts.cpu().view(self.P.B, -1).tolist() == self.counts, what + ": counts"

    def reserve(self, T, new=None, own_all=False, what=""):
        n = [T] * self.P.B if new is None else [min(max(x, 0), T) for x in new]
        want, lack = O.reserve(self.tables, self.refs, self.held, n, self.page, own_all)
        pairs, done = self.C.compactor_pages_reserve(self.cache, self.dev_refs, T, new_tokens=_new(new), own_all=own_all)
        assert done.tolist() == [len(want), lack] and [tuple(x) for x in pairs[:len(want)].tolist()] == want, what
        self.same(what)
        self.copy(pairs, done, want)
        return want, lack


COUNTS = (40, 0, 17, 33, 100, 16, 64, 96)


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("page,layout,state", [(16, "token", True), (7, "head", True), (24, "layer", False), (1, "token", True), (64, "head", True)])
@pytest.mark.parametrize("own_all", [False, True])
@pytest.mark.parametrize("T,new", [(0, None), (1, None), (5, [5, 0, 3, 1, 9, -2]), (90, None)])
def test_reserve(C, mx, page, layout, state, own_all, T, new):
    W = World(C, _counts(6, 2, 3, *COUNTS), page=page, entries=-(-160 // page), spare=6 * 100, mx=mx, layout=layout, state=state)
    W.share([(0, 1, 2), (0, 2, 1), (4, 5, -(-100 // page)), (4, 3, 1)])
    W.load()
    W.reserve(T, new, own_all)
    W.reserve(T, new, own_all, "again")                    # now everything is there


@pytest.mark.parametrize("samples", [2, 3, 8])
@pytest.mark.parametrize("new", [None, "some"])
def test_reserve_samples_of_a_prompt(C, samples, new):
    """All write to the page that they share: the last one keeps it where all are there."""
    B = 4 * samples
    W = World(C, [[[35 + 16 * (b // samples)] * 4] for b in range(B)], page=16, entries=8, spare=5 * B)
    W.share([(b - b % samples, b, 6) for b in range(B) if b % samples])
    W.load()
    W.reserve(1, None if new is None else [b % 3 for b in range(B)])
    own = torch.stack([W.P.tables[b, 2 + b // samples] for b in range(B)])
    if new is None:
        assert own.unique().numel() == B


def test_reserve_too_few_pages(C):
    W = World(C, [[[32]] for _ in range(6)], page=16, entries=4, spare=5, foreign=1)
    W.load()
    want, lack = W.reserve(20)                              # 12 wanted, 4 free
    assert lack == 8 and not want
    want, lack = W.reserve(1, [1, 0, 1, 0, 1, 1])
    assert lack == 0
    want, lack = W.reserve(1, [0, 1, 0, 0, 0, 0])
    assert lack == 1


def test_reserve_odd_tables(C):
    """Entries that are no pages, a page that a request names twice, counts outside the table, tables that end."""
    W = World(C, _counts(5, 1, 2, 40, 33, 64, 50, 16, 16, 5, 200, 10 ** 6, -4), page=16, entries=6, spare=40)
    W.counts[4][1] = -4
    W.tables[0][1], W.tables[0][4], W.tables[1][5] = -7, 10 ** 9, len(W.refs)
    W.share([(2, 3, 1)])
    a = W.tables[1][2]
    W.refs[W.tables[1][3]] -= 1
    W.tables[1][3] = a
    W.refs[a] += 1
    W.load()
    for own_all in (False, True):
        W.reserve(30, [3, 30, 30, 17, 1], own_all)


@pytest.mark.parametrize("B,L,H,entries,own_all", [(1, 1, 1, 1, False), (130, 1, 2, 70, True), (1100, 1, 1, 4, False), (3, 40, 9, 300, True), (2000, 1, 1, 3, True)])
def test_reserve_many(C, B, L, H, entries, own_all):
    """More entries, requests and pages than a pass of the plan takes."""
    rng = np.random.default_rng(B)
    counts = rng.integers(0, entries * 2, (B, L, H)).tolist()
    W = World(C, counts, page=2, entries=entries, spare=max(0, 2 * B * entries - B * (entries // 2)), layout="head")
    W.share([(b - b % 4, b, int(rng.integers(0, entries + 1))) for b in range(B) if b % 4])
    W.load()
    W.reserve(5, rng.integers(-1, 7, B).tolist(), own_all)


@pytest.mark.parametrize("N", [70, 4095, 4096, 4097, 4103, 4112, 20011, 20480, 61000])
@pytest.mark.parametrize("lead", [0, 1])
@pytest.mark.parametrize("free", ["last", "few", "half", "too few"])
def test_reserve_pools(C, N, lead, free):
    """Free pages anywhere in pools of all sizes, counts of references that begin anywhere."""
    rng = np.random.default_rng(N)
    wants = 40
    refs = np.ones(N, np.int64)
    refs[{"last": np.arange(N - wants, N), "few": rng.permutation(N)[:wants + 3], "half": rng.permutation(N)[:max(N // 2, wants)],
          "too few": rng.permutation(N)[:wants - 1]}[free]] = 0
    k = torch.empty(N, 1, 1, 1, 128, dtype=torch.bfloat16, device=DEV)
    tables = [[-1, -1, -1] for _ in range(wants)]
    cache = C.Cache(k, k.clone(), torch.tensor(tables, dtype=torch.int32, device=DEV), torch.zeros(wants, 1, 1, dtype=torch.int32, device=DEV))
    dev = torch.tensor([9] * lead + refs.tolist(), dtype=torch.int32, device=DEV)[lead:]
    r = refs.tolist()
    want, lack = O.reserve(tables, r, [[0]] * wants, [1] * wants, 1, False)
    pairs, done = C.compactor_pages_reserve(cache, dev, 1)
    assert done.tolist() == [len(want), lack] and cache.tables.tolist() == tables and dev.tolist() == r


@pytest.mark.parametrize("B,L,H,entries", [(1, 1, 1, 1), (6, 2, 3, 10), (64, 1, 4, 130), (300, 1, 1, 70), (5, 9, 8, 65), (2000, 1, 2, 5)])
@pytest.mark.parametrize("state", [True, False])
def test_fork(C, B, L, H, entries, state):
    rng = np.random.default_rng(B)
    W = World(C, rng.integers(0, entries * 2, (B, L, H)).tolist(), page=2, entries=entries, state=state)
    W.share([(b - 1, b, entries // 2) for b in range(1, B, 3)])
    W.tables[0][0] = 10 ** 8
    W.refs = [0] * len(W.refs)
    for t in W.tables:
        for p in t:
            if 0 <= p < len(W.refs):
                W.refs[p] += 1
    W.load()
    for parents in (rng.permutation(B), rng.integers(0, B, B), rng.integers(-2, B + 2, B), np.zeros(B, int)):
        parents = [int(x) for x in parents]
        O.fork(W.tables, W.refs, [W.counts] + ([W.seen] if state else []), parents)
        C.compactor_pages_fork(W.cache, W.dev_refs, torch.tensor(parents, dtype=torch.int32, device=DEV))
        W.same()
        assert W.P.seen.cpu().view(B, -1).tolist() == W.seen


@pytest.mark.parametrize("B,L,H,entries", [(1, 1, 1, 1), (6, 2, 3, 10), (64, 1, 4, 130), (5, 40, 9, 600), (2000, 1, 2, 5)])
def test_release_and_compact(C, B, L, H, entries):
    rng = np.random.default_rng(B)
    W = World(C, rng.integers(0, entries * 2, (B, L, H)).tolist(), page=2, entries=entries, spare=30)
    W.share([(b - 1, b, entries // 2) for b in range(1, B, 3)])
    W.load()
    W.reserve(3)                                           # pages that no token is in yet are given back too
    for finished in (None, rng.random(B) < 0.4, np.zeros(B), np.ones(B)):
        f = None if finished is None else [int(x) * (b + 1) for b, x in enumerate(finished)]
        O.release(W.tables, W.refs, [W.counts, W.seen], 2, f or [0] * B)
        C.compactor_pages_release(W.cache, W.dev_refs, finished=_new(f))
        W.same("release")
        assert W.P.seen.cpu().view(B, -1).tolist() == W.seen
        before = [list(t) for t in W.tables]
        want, n = O.compact(W.tables, W.refs)
        pairs, done = C.compactor_pages_compact(W.cache, W.dev_refs)
        assert done.tolist() == [len(want), n] and [tuple(x) for x in pairs[:len(want)].tolist()] == want
        W.same("compact")
        W.copy(pairs, done, want)
        assert all(r > 0 for r in W.refs[:n]) and not any(W.refs[n:]) and (not want or before != W.tables or W.refs)


@pytest.mark.parametrize("N", [1, 2, 15, 16, 17, 4095, 4096, 4097, 16384, 16391, 20011, 61000])
@pytest.mark.parametrize("share", [0.0, 0.02, 0.5, 1.0])
def test_compact_pools(C, N, share):
    rng = np.random.default_rng(N)
    refs = (rng.random(N) < share) * rng.integers(1, 5, N)
    k = torch.zeros(N, 1, 1, 1, 128, dtype=torch.bfloat16, device=DEV)
    k.view(N, 128)[:, 0] = torch.arange(N) % 256
    k.view(N, 128)[:, 1] = torch.arange(N) // 256
    tables = rng.permutation(N)[:max(1, N // 2)].reshape(1, -1)
    cache = C.Cache(k, k.clone(), torch.tensor(tables, dtype=torch.int32, device=DEV), torch.ones(1, 1, 1, dtype=torch.int32, device=DEV))
    t, r = tables.tolist(), [int(x) for x in refs]
    want, n = O.compact(t, r)
    dev = torch.tensor(refs, dtype=torch.int32, device=DEV)
    was = k.clone()
    pairs, done = C.compactor_pages_compact(cache, dev)
    C.compactor_pages_copy(cache, pairs, done)
    for a, b in want:
        was[b] = was[a]
    assert done.tolist() == [len(want), n] and cache.tables.tolist() == t and dev.tolist() == r
    assert torch.equal(k, was) and torch.equal(cache.v_pages, was)


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("L,H,page,layout", [(1, 1, 1, "token"), (3, 5, 7, "head"), (2, 8, 16, "layer"), (32, 8, 16, "token"), (1, 1, 3, "head"), (2, 3, 128, "layer")])
def test_copy(C, mx, L, H, page, layout):
    """Only the first pairs, those with a page that is not there passed over; a pool inside a larger one."""
    W = World(C, _counts(3, L, H, 40, 5), page=page, mx=mx, layout=layout, spare=40)
    W.load()
    N = W.P.pages
    pairs = torch.tensor([[0, N - 1], [1, N - 2], [-1, 3], [4, N], [5, N - 3], [6, N - 4], [2, N - 5]], dtype=torch.int32, device=DEV)
    for n, want in ((0, []), (5, [(0, N - 1), (1, N - 2), (5, N - 3)]), (100, [(0, N - 1), (1, N - 2), (5, N - 3), (6, N - 4), (2, N - 5)]), (-3, [])):
        W.copy(pairs, torch.tensor([n, 0], dtype=torch.int32, device=DEV), want)
    if not mx:
        wide = torch.randn(N, L + 1, page, H + 2, 136, device=DEV).to(torch.bfloat16)
        part = wide[:, 1:, :, 1:H + 1, 8:]
        cache = C.Cache(part, wide.clone()[:, 1:, :, 1:H + 1, 8:], W.P.tables, W.P.counts)
        was = wide.clone()
        C.compactor_pages_copy(cache, pairs, torch.tensor([2, 0], dtype=torch.int32, device=DEV))
        for a, b in ((0, N - 1), (1, N - 2)):
            was[b, 1:, :, 1:H + 1, 8:] = was[a, 1:, :, 1:H + 1, 8:]
        assert torch.equal(wide, was)


def test_copy_far_into_a_large_pool(C):
    """Pages beyond 2^32 bytes."""
    page, H = 64, 8
    pages = (2 ** 31 + 2 ** 28) // (page * H * 128)
    pool = torch.empty(pages, 1, page, H, 128, dtype=torch.bfloat16, device=DEV)
    pool[:4] = torch.randn(4, 1, page, H, 128, device=DEV).to(torch.bfloat16)
    cache = C.Cache(pool, pool, torch.zeros(1, 1, dtype=torch.int32, device=DEV), torch.zeros(1, 1, H, dtype=torch.int32, device=DEV))
    pairs = torch.tensor([[0, pages - 1], [3, pages - 7]], dtype=torch.int32, device=DEV)
    C.compactor_pages_copy(cache, pairs, torch.tensor([2, 0], dtype=torch.int32, device=DEV))
    assert torch.equal(pool[pages - 1], pool[0]) and torch.equal(pool[pages - 7], pool[3])


@pytest.mark.parametrize("mx", [False, True])
def test_samples_and_beams_as_they_would_be_used(C, mx):
    """Samples of prompts share pages, go apart as they append, are reordered, end and are pushed together: attention to a sample is at each step that to
    a cache of its own that was given the same tokens."""
    H, G, B, samples = 2, 2, 6, 3
    W = World(C, [[[37 if b < 3 else 50] * H] for b in range(B)], page=16, entries=8, spare=60, mx=mx)
    W.share([(b - b % samples, b, 4) for b in range(B) if b % samples])
    W.load()
    P, cache, refs = W.P, W.cache, W.dev_refs
    append, attend, copy = ((C.compactor_mx_append, C.compactor_mx_attention, C.compactor_mx_pages_copy) if mx else
                            (C.compactor_cache_append, C.compactor_cache_attention, C.compactor_pages_copy))
    make = X.Paged if mx else U.Paged
    alone = make(C, DEV, [[[0] * H] for _ in range(B)], page=16, room=128)
    other = alone.mx_handle() if mx else alone.handle()

    def put():
        for n in X.ROWS if mx else ("k", "v"):          # the same rows, request by request
            for b in range(B):
                for i in range(W.entries):
                    if int(P.tables[b, i]) >= 0:
                        getattr(alone, n)[int(alone.tables[b, i])] = getattr(P, n)[int(P.tables[b, i])]
        alone.counts.copy_(P.counts), alone.seen.copy_(P.seen)

    put()
    g = torch.Generator(device=DEV)
    g.manual_seed(3)

    def step():
        k, v = (torch.randn(B, 1, 1, H, 128, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
        q = torch.randn(B, 1, 1, H * G, 128, generator=g, device=DEV).to(torch.bfloat16)
        pairs, done = C.compactor_pages_reserve(cache, refs, 1)
        copy(cache, pairs, done)
        assert int(done[1]) == 0
        got = []
        for c in (cache, other):
            append(c, k, v)
            got.append(attend(c, q, want_lse=True))
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])

    for _ in range(13):
        step()
    parents = torch.tensor([1, 1, 0, 5, 5, 3], dtype=torch.int32, device=DEV)
    C.compactor_pages_fork(cache, refs, parents)
    put()
    for _ in range(4):
        step()
    finished = torch.tensor([0, 1, 0, 0, 0, 1], dtype=torch.int32, device=DEV)
    C.compactor_pages_release(cache, refs, finished=finished)
    pairs, done = C.compactor_pages_compact(cache, refs)
    copy(cache, pairs, done)
    assert int(done[0]) > 0 and not refs[int(done[1]):].any()
    alone.counts.mul_(1 - finished.view(B, 1, 1)), alone.seen.mul_(1 - finished.view(B, 1, 1))
    for _ in range(3):
        step()
    named = P.tables[P.tables >= 0]
    count = torch.bincount(named.long(), minlength=P.pages)
    assert torch.equal(count[:int(refs.numel())] > 0, refs > 0) or int((refs > 0).sum()) == int((count > 0).sum()) + 2


def test_a_captured_step(C):
    """Reserve, copy and append in one graph, replayed as the cache grows, against the eager calls on a copy, on a stream of its own."""
    def make():
        W = World(C, [[[37] * 2] for _ in range(4)], page=16, entries=12, spare=60)
        W.share([(0, b, 3) for b in range(1, 4)])
        W.load()
        return W

    a, b = make(), make()
    k, v = (torch.randn(4, 1, 5, 2, 128, device=DEV).to(torch.bfloat16) for _ in range(2))
    new = torch.ones(4, dtype=torch.int32, device=DEV)
    parents = torch.arange(4, dtype=torch.int32, device=DEV)
    finished = torch.zeros(4, dtype=torch.int32, device=DEV)

    def step(W, stream=None):
        C.compactor_pages_fork(W.cache, W.dev_refs, parents, stream=stream)
        pairs, done = C.compactor_pages_reserve(W.cache, W.dev_refs, 5, new_tokens=new, stream=stream)
        C.compactor_pages_copy(W.cache, pairs, done, stream=stream)
        C.compactor_cache_append(W.cache, k, v, new_tokens=new, stream=stream)
        C.compactor_pages_release(W.cache, W.dev_refs, finished=finished, stream=stream)
        pairs, moved = C.compactor_pages_compact(W.cache, W.dev_refs, stream=stream)
        C.compactor_pages_copy(W.cache, pairs, moved, stream=stream)
        return done, moved

    step(make())
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        got = step(a)
    for i, (n, p, f) in enumerate([([1, 1, 1, 1], [0, 1, 2, 3], 0), ([5, 0, 2, 1], [0, 0, 2, 3], 0), ([5, 5, 5, 5], [3, 2, 1, 0], 0), ([0, 0, 0, 0], [0, 1, 2, 3], 0),
                                   ([1, 5, 0, 3], [1, 1, 1, 3], 1), ([4, 4, 4, 4], [0, 1, 2, 2], 0)]):
        new.copy_(torch.tensor(n, dtype=torch.int32)), parents.copy_(torch.tensor(p, dtype=torch.int32)), finished.zero_()
        finished[2] = f
        graph.replay()
        side.wait_stream(torch.cuda.current_stream())
        want = step(b, side)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(a.dev_refs, b.dev_refs), i
        assert torch.equal(a.P.tables, b.P.tables), i
        U.same_pool(a.P, b.P.snapshot(), "replay %d" % i)
