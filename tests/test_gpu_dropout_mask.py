"""GPU: the mask of halo_dropout."""
import numpy as np
import pytest
import torch

from oracle import adapters_oracle as orc
from paper_2501_02625_amd import binding
from tests import gpu_util as gu

pytestmark = pytest.mark.gpu


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
