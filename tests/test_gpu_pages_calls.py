"""Pages of caches of the most requests that the calls take, and every count of references after a pool has been pushed together."""
import numpy as np
import pytest
import torch

from oracle import pages_oracle as O
from tests import gpu_util as GU
from tests.test_gpu_cache import DEV, _new
from tests.test_gpu_pages import World

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def C():
    return GU.binding()


@pytest.mark.parametrize("B,H,entries", [(8192, 2, 5), (16383, 1, 3), (16384, 2, 4)])
def test_the_most_requests(C, B, H, entries):
    rng = np.random.default_rng(B)
    W = World(C, rng.integers(0, entries * 2, (B, 1, H)).tolist(), page=2, entries=entries, spare=B * entries)
    W.share([(b - 1, b, entries // 2) for b in range(1, B, 3)])
    W.load()
    W.reserve(2, rng.integers(0, 3, B).tolist(), what="reserve")
    for parents in (rng.permutation(B), rng.integers(-2, B + 2, B)):
        parents = [int(x) for x in parents]
        O.fork(W.tables, W.refs, [W.counts, W.seen], parents)
        C.compactor_pages_fork(W.cache, W.dev_refs, _new(parents))
        W.same("fork")
        assert W.P.seen.cpu().view(B, -1).tolist() == W.seen
    finished = [int(x) for x in rng.random(B) < 0.4]
    O.release(W.tables, W.refs, [W.counts, W.seen], 2, finished)
    C.compactor_pages_release(W.cache, W.dev_refs, finished=_new(finished))
    W.same("release")
    want, n = O.compact(W.tables, W.refs)
    pairs, done = C.compactor_pages_compact(W.cache, W.dev_refs)
    assert done.tolist() == [len(want), n] and [tuple(x) for x in pairs[:len(want)].tolist()] == want
    W.same("compact")


@pytest.mark.parametrize("mx", [False, True])
def test_counts_of_references_after_everything(C, mx):
    """Samples that go apart, are reordered, end and are pushed together: each page is counted as often as the tables name it, and those that
    somebody else holds are counted once wherever they have moved."""
    B, samples = 12, 4
    W = World(C, [[[37 + 16 * (b // samples)] * 2] for b in range(B)], page=16, entries=9, spare=90, mx=mx, foreign=5)
    W.share([(b - b % samples, b, 7) for b in range(B) if b % samples])
    W.load()
    N = W.P.pages
    foreign = [p for p in range(N) if W.refs[p] == 1 and not any(p in t for t in W.tables)]
    assert len(foreign) == 5
    rng = np.random.default_rng(2)

    def counted():
        named = W.P.tables[(W.P.tables >= 0) & (W.P.tables < N)].long()
        want = torch.bincount(named, minlength=N)
        want[torch.tensor(foreign, device=DEV)] += 1
        assert torch.equal(W.dev_refs.long(), want)

    moved = 0
    for i in range(5):
        new = rng.integers(0, 20, B).tolist()
        want, lack = W.reserve(20, new, own_all=i == 3)
        assert lack == 0
        counted()
        W.P.counts += torch.tensor(new, dtype=torch.int32, device=DEV).view(B, 1, 1)
        parents = rng.integers(0, B, B).tolist()
        C.compactor_pages_fork(W.cache, W.dev_refs, _new(parents))
        counted()
        C.compactor_pages_release(W.cache, W.dev_refs, finished=_new((rng.random(B) < 0.3).astype(int).tolist()))
        counted()
        pairs, done = C.compactor_pages_compact(W.cache, W.dev_refs)
        n = int(done[0])
        to = {a: z for a, z in pairs[:n].tolist()}
        foreign = [to.get(p, p) for p in foreign]
        moved += n
        counted()
        assert not W.dev_refs[int(done[1]):].any() and bool((W.dev_refs[:int(done[1])] > 0).all())
        (C.compactor_mx_pages_copy if mx else C.compactor_pages_copy)(W.cache, pairs, done)
        # what the plain lists go on from
        W.tables, W.refs = W.P.tables.tolist(), W.dev_refs.tolist()
        W.counts = W.P.counts.cpu().view(B, -1).tolist()
        W.held = [[min(max(x, 0), W.P.capacity) for x in b] for b in W.counts]
        W.rows = {name: getattr(W.P, name).clone() for name in W.rows}
    assert moved > 0
