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


def test_store_of_little_in_large_tables(C):
    """4096 heads whose tables have room for 2^18 tokens each, which nearly none of them holds: as request by request with tables that just suffice."""
    B, L, H, page = 64, 8, 8, 16
    lengths = [3001, 1025] + [(17 * b) % 41 for b in range(2, B)]
    need = [-(-n // page) for n in lengths]
    N, g = sum(need) + 3, torch.Generator(device=DEV)
    g.manual_seed(1)
    k, v = (torch.randn(N, L, H, page, 128, generator=g, device=DEV).to(torch.bfloat16).transpose(2, 3) for _ in range(2))
    mass = torch.rand(N, L, H, page, generator=g, device=DEV)
    positions = torch.randint(0, 1 << 20, mass.shape, generator=g, device=DEV, dtype=torch.int32)
    order, tables, at = torch.randperm(N, generator=g, device=DEV).to(torch.int32), torch.full((B, 1 << 14), -1, dtype=torch.int32, device=DEV), 0
    for b in range(B):
        tables[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
    counts = torch.tensor(lengths, dtype=torch.int32, device=DEV).view(B, 1, 1).expand(B, L, H).contiguous()
    counts[0, 3, 2], counts[1, 7, 7], counts[5, 0, 0] = 2049, 0, -3
    seen = counts + 5

    def made():
        rows = [torch.full((N, L, page, H, 64), 9, dtype=torch.uint8, device=DEV) for _ in range(2)]
        scales = [torch.full((N, L, H, page, 4), 9, dtype=torch.uint8, device=DEV) for _ in range(2)]
        return rows + scales + [torch.full_like(counts, 7), torch.full_like(counts, 7), torch.full_like(mass, 7.0), torch.full_like(positions, 7)]

    got, want = made(), made()
    C.compactor_mx_store(C.MxCache(*got[:4], tables, *got[4:]), C.Cache(k, v, tables, counts, seen, mass, positions))
    for b in range(B):
        some = tables[b:b + 1, :max(1, need[b])].contiguous()
        C.compactor_mx_store(C.MxCache(*want[:4], some, want[4][b:b + 1], want[5][b:b + 1], *want[6:]),
                             C.Cache(k, v, some, counts[b:b + 1], seen[b:b + 1], mass, positions))
    for x, y in zip(got, want):
        assert torch.equal(x, y)
    assert torch.equal(got[4], counts.clamp(min=0)) and torch.equal(got[5], seen)
    rows = C.compactor_mx_read(C.MxCache(*got[:4], tables, *got[4:]), 3001, first=0)
    # Of a group whose largest magnitude is m 2^k a number is off by 2^(k - 2) at most: with m < 1.75 the scale is 2^(k - 2), the widest step, 4 to 6, 2 of it, and 7
    # becomes 6; else the scale is 2^(k - 1), all numbers are up to 4 of it and the widest step is 1.  As m >= 1 that is a quarter of the largest.
    for t, pool in zip(rows, (k, v)):
        plain = pool[tables[0, :need[0]].long()].permute(1, 0, 2, 3, 4).reshape(L, -1, H, 128)[:, :3001].float()
        there = (torch.arange(3001, device=DEV).view(1, -1, 1) < counts[0].view(L, 1, H)).unsqueeze(-1)
        top = plain.view(L, 3001, H, 4, 32).abs().amax(-1, keepdim=True).expand(L, 3001, H, 4, 32).reshape(plain.shape)
        off = (t[0].float() - plain).abs()
        assert float((off - top / 4).masked_fill(~there, -1.0).max()) <= 0.0 and not t[0].masked_fill(there, 0.0).any()
