"""GPU: the mask of halo_dropout in every form of the call, and of a matrix of more elements than a launch has threads in one dimension."""
import numpy as np
import pytest
import torch

from oracle import adapters_oracle as orc
from paper_2501_02625_amd import binding
from tests import gpu_util as gu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(3, 8), (65, 520), (129, 1000)])
@pytest.mark.parametrize("p", [0.1, 0.5, 1.0])
def test_one_mask_for_the_branch_and_its_gradient(dtype, rows, cols, p):
    """Values and a residual that tell which elements were kept: with a residual, without, into the input, and the gradient's call."""
    seed, offset = 2**63 + rows, 2**40 + cols
    keep = gu.to_dev(orc.keep_mask(rows, cols, p, seed, offset))
    x = torch.full((rows, cols), 8.0, dtype=dtype, device=gu.DEV)
    res = torch.full((rows, cols), 1.0, dtype=dtype, device=gu.DEV)
    a, b = x.clone(), res.clone()
    for y in (binding.halo_dropout(x, p, seed, offset, residual=res), binding.halo_dropout(a, p, seed, offset, residual=res, out=a),
              binding.halo_dropout(x, p, seed, offset, residual=b, out=b)):
        assert torch.equal(y != 1.0, keep)
    assert torch.equal(binding.halo_dropout(x, p, seed, offset) != 0.0, keep)


@pytest.mark.parametrize("residual", [False, True])
def test_inner_products_of_the_branch_and_its_gradient(residual):
    """<g, drop(x)> = <drop(g), x>: the same products, each with the one factor, in fp32 up to a rounding of each element (2^-24, and
    another one with the residual, which is taken off again)."""
    n = torch.Generator(device=gu.DEV).manual_seed(3)
    x, g, res = (torch.randn((190, 1000), generator=n, device=gu.DEV) for _ in range(3))
    y = binding.halo_dropout(x, 0.3, 17, 18, residual=res if residual else None).double()
    if residual:
        y -= res.double()
    left, right = (g.double() * y).sum(), (binding.halo_dropout(g, 0.3, 17, 18).double() * x.double()).sum()
    size = (g.double() * (y.abs() + (res.double().abs() if residual else 0.0))).abs().sum()
    assert abs(left - right) <= 4 * 2.0 ** -24 * size


def test_more_elements_than_one_dimension_of_a_launch_has_threads():
    """2^36 elements and some: 137 GB, in place."""
    rows, cols = (1 << 14) + 3, 1 << 22
    if torch.cuda.mem_get_info()[0] < rows * cols * 2 + (4 << 30):
        pytest.skip("not enough free memory on this card")
    x = torch.ones((rows, cols), dtype=torch.bfloat16, device=gu.DEV)
    y = binding.halo_dropout(x, 0.5, 21, 22, out=x)
    for row in (0, 1, rows // 2, rows - 4, rows - 3, rows - 2, rows - 1):
        for at in (0, cols // 2, cols - 64):
            # the oracle's mask of 64 columns of one row: its counter is (column / 8, row)
            groups = np.arange(at // 8, at // 8 + 8, dtype=np.uint64)
            words = orc.philox4x32_10([groups, np.full(8, row, dtype=np.uint64), np.full(8, 22, dtype=np.uint64),
                                       np.zeros(8, dtype=np.uint64)], [21, 0])
            halves = [h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))]
            keep = np.stack(halves, axis=-1).reshape(64) >= 32768
            assert np.array_equal(y[row, at:at + 64].float().cpu().numpy(), np.where(keep, 2.0, 0.0)), (row, at)
    del x, y
    torch.cuda.empty_cache()
