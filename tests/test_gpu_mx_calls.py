"""Calls of a cache in 4 bits that hold little of what their tables have room for, or one long context among many short ones."""
import pytest
import torch

from tests import cache_util as U
from tests import gpu_util as GU
from tests import mx_util as X
from tests.test_gpu_cache import DEV, _queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def C():
    return GU.binding()


@pytest.mark.parametrize("page", [16, 24])
@pytest.mark.parametrize("G,T", [(4, 1), (4, 5), (16, 4)])
def test_attention_of_a_long_head_among_hundreds(C, page, G, T):
    """480 heads, nearly all of one step or none, and a few that are cut into many fragments."""
    P = X.Paged(C, DEV, [[[34001, 40, 0, 5000, 129, 1, 128, 16385]]], page=page)
    B = 60
    tables = torch.full((B, P.per), -1, dtype=torch.int32, device=DEV)
    tables[7] = P.tables[0]
    counts, seen = (torch.zeros(B, 1, 8, dtype=torch.int32, device=DEV) for _ in range(2))
    counts[7] = P.counts[0]
    cache = C.MxCache(P.k4, P.v4, P.k_scales, P.v_scales, tables, counts, seen, P.mass, P.positions)
    q = torch.zeros(B, 1, T, 8 * G, 128, dtype=torch.bfloat16, device=DEV)
    q[7:8] = _queries(P, T, 8 * G)
    before = P.snapshot()
    out, lse = C.compactor_mx_attention(cache, q, accumulate=True, want_lse=True)
    torch.cuda.synchronize()
    assert torch.isneginf(lse[:7]).all() and torch.isneginf(lse[8:]).all() and not out[:7].any() and not out[8:].any()
    U.check_attention(P, q[7:8], None, 128 ** -0.5, 0.0, out[7:8], lse[7:8], before, True)
