"""GPU: pools without in-features or without out-features.  The C ABI does nothing for them, so the binding has no results to return."""
import pytest
import torch

from paper_2501_02625_amd import binding
from tests import gpu_util as gu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("b", [0, 5])
@pytest.mark.parametrize("m,n", [(64, 0), (0, 64), (0, 0)])
def test_a_pool_of_no_width_is_refused(b, m, n):
    zeros = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16, device=gu.DEV)
    X, E, U, V = zeros(b, m), zeros(b, n), zeros(3, 8, m), zeros(3, n, 8)
    of, T = torch.zeros(b, dtype=torch.int32, device=gu.DEV), torch.zeros((b, 8), device=gu.DEV)
    Y, EX = torch.full((b, n), 3.0, dtype=torch.bfloat16, device=gu.DEV), torch.full((b, m), 3.0, dtype=torch.bfloat16, device=gu.DEV)
    with pytest.raises(AssertionError):
        binding.halo_adapters_fwd(X, U, V, of, base=zeros(b, n), Y=Y)
    with pytest.raises(AssertionError):
        binding.halo_adapters_bwd(E, X, T, U, V, of, base=zeros(b, m), EX=EX)
    assert (Y == 3).all() and (EX == 3).all()
