"""Norms and rotation in calls that nothing else makes: so many layers that their weights pass 2^31 numbers; queries rotated in place beside the append."""
import pytest
import torch

from tests import cache_util as U
from tests import gpu_util as GU
from tests import mx_util as X
from tests.test_gpu_cache import DEV, _counts, _new
from tests.test_gpu_rotate import EPS, _rotation, _rows, _separately, _together, _Twins

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def C():
    return GU.binding()


def test_weights_of_more_layers_than_32_bits_reach(C):
    """The last layers have rows and weights of their own, and get what they get alone."""
    L, some = (1 << 24) + 3, 5
    weights = torch.ones(L, 128, device=DEV)
    weights[-some:] = 0.5 + torch.rand(some, 128, device=DEV)
    freqs = 10000.0 ** (-torch.arange(64, device=DEV, dtype=torch.float64) / 64)
    k = torch.ones(1, L, 1, 1, 128, dtype=torch.bfloat16, device=DEV)
    k[:, -some:] = _rows((1, some, 1, 1, 128), 1)
    at = torch.tensor([77], dtype=torch.int32, device=DEV)
    _, got, _ = C.compactor_rotate(C.Rotation(freqs, k_norm=weights, eps=EPS), None, k, at, k_out=k.clone())
    _, want, _ = C.compactor_rotate(C.Rotation(freqs, k_norm=weights[-some:].contiguous(), eps=EPS), None, k[:, -some:].contiguous(), at)
    assert torch.equal(U.bits(got[:, -some:]), U.bits(want))
    assert torch.equal(U.bits(got[:, :1]), U.bits(got[:, L // 2:L // 2 + 1]))


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("T,new", [(1, None), (1, [1, 0, 1]), (5, [5, 0, 3]), (9, None), (65, [0, 65, 64]), (130, [130, 3, 129])])
@pytest.mark.parametrize("G,rotary,interleaved,page,layout", [(1, 128, False, 16, "token"), (4, 64, True, 24, "head"), (7, 96, False, 7, "layer")])
def test_one_layer_in_place(C, mx, T, new, G, rotary, interleaved, page, layout):
    """Queries that become the rotated ones where they lie, of one layer of a cache of three: what that layer gets, bit by bit, and nothing else."""
    twins = _Twins(C, mx, _counts(3, 3, 2, 40, 0, 17, 33, 100), page=page, layout=layout, room=90)
    for P in (twins.a, twins.b):
        P.tables[1, (40 + T // 2) // page] = -1
        P.seen.copy_((torch.arange(18) * 1000).view(3, 3, 2))
    rotation = _rotation(C, rotary, interleaved, layers=3)
    q, k, v = _rows((3, 3, T, 2 * G, 128), 1), _rows((3, 3, T, 2, 128), 2), _rows((3, 3, T, 2, 128), 3)
    a, b = twins.cache(twins.a), twins.cache(twins.b)
    want = q.clone()
    rotated = _separately_one(C, twins.b, b, rotation, q, k, v, new, 1)
    n = torch.full((3,), T) if new is None else torch.tensor(new).clamp(0, T)
    real = (torch.arange(T) < n.view(3, 1)).to(DEV).view(3, T, 1, 1)
    want[:, 1] = torch.where(real, rotated, q[:, 1])
    got = q.clone()
    back = _together(C, a)(a.layer(1), rotation.layer(1), k[:, 1:2], v[:, 1:2], got[:, 1:2], new_tokens=_new(new), q_out=got[:, 1:2])
    assert back.data_ptr() == got[:, 1:2].data_ptr()
    assert torch.equal(U.bits(got), U.bits(want))
    twins.same()


class _Layer:
    """One layer of a paged cache, as _separately takes it."""

    def __init__(self, P, l):
        self.seen = P.seen[:, l:l + 1]


def _separately_one(C, P, cache, rotation, q, k, v, new, l):
    at = slice(l, l + 1)
    return _separately(C, _Layer(P, l), cache.layer(l), rotation.layer(l), *(t[:, at].contiguous() for t in (q, k, v)), new)[:, 0]


@pytest.mark.parametrize("mx", [False, True])
def test_a_captured_step_in_place(C, mx):
    """The queries' buffer is rotated where it lies and attention reads it there; replayed as the cache grows, against the eager calls on a copy."""
    counts = _counts(3, 1, 4, 100, 90, 33, 140)
    twins = _Twins(C, mx, counts, page=16, room=80)
    rotation = _rotation(C)
    k, v = (torch.zeros(3, 1, 1, 4, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    q, other = (torch.zeros(3, 1, 1, 16, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    new = torch.ones(3, dtype=torch.int32, device=DEV)
    a, b = twins.cache(twins.a), twins.cache(twins.b)
    attend = C.compactor_mx_attention if mx else C.compactor_cache_attention

    def step(cache, x):
        _together(C, cache)(cache, rotation, k, v, x, new_tokens=new, q_out=x)
        return attend(cache, x, new_tokens=new, accumulate=True)[0]

    step(twins.cache((X.Paged if mx else U.Paged)(C, DEV, counts, page=16, room=80)), q)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(a, q)
    g = torch.Generator(device=DEV)
    g.manual_seed(8)
    for i in range(6):
        for t in (k, v, q):
            t.copy_(torch.randn(t.shape, generator=g, device=DEV))
        other.copy_(q)
        given = q.clone()
        new.copy_(torch.tensor([1, i % 2, 1 if i < 3 else 0], dtype=torch.int32))
        graph.replay()
        want = step(b, other)
        torch.cuda.synchronize()
        assert torch.equal(U.bits(got), U.bits(want)) and torch.equal(U.bits(q), U.bits(other)), i
        for r in range(3):
            assert torch.equal(q[r], given[r]) == (int(new[r]) == 0), i          # padding rows stay, the others do not
        twins.same("replay %d" % i)
