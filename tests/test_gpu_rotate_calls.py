"""Norms and rotation in calls that nothing else makes: so many layers that their weights pass 2^31 numbers."""
import pytest
import torch

from tests import cache_util as U
from tests import gpu_util as GU
from tests.test_gpu_cache import DEV
from tests.test_gpu_rotate import EPS, _rows

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
