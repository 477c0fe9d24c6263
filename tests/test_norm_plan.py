"""CPU test of the workspace that the norm's gradient asks for: as many parts of the rows as its launch writes, and one, which nothing is
written to, where few rows take one launch."""
import ctypes
import os

import pytest

from paper_2501_02625_amd import _build, binding

BF16, F32 = binding.HALO_BF16, binding.HALO_F32


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_build.LIB_PATH):
        _build.build()
    return binding.load_library()


# rows, columns, type, parts.  Up to 1024 columns a workgroup has 32, 16, 8 or 4 rows at once; it is one of 512 at most, beyond 4096
# columns one of 256; beyond 8192 (fp32) and 16384 (bf16) parts are of 16 rows at least, and 2048 workgroups of 512 columns at most.
@pytest.mark.parametrize("rows,cols,dt,parts", [
    (1, 1, BF16, 1), (256, 500, F32, 1), (257, 500, F32, 65), (512, 513, BF16, 1), (513, 513, BF16, 129), (512, 14336, BF16, 1), (512, 32768, F32, 1),
    (10000, 64, F32, 313), (20000, 64, BF16, 512), (4000, 128, BF16, 250), (4000, 256, BF16, 500), (5000, 256, BF16, 512), (2048, 1024, F32, 512),
    (513, 1025, BF16, 512), (8192, 4096, BF16, 512), (8192, 4097, BF16, 256), (2048, 8192, F32, 256), (513, 8200, BF16, 256), (8192, 16384, BF16, 256),
    (513, 8200, F32, 33), (8192, 8200, F32, 120), (600, 16385, BF16, 38), (1 << 20, 32768, BF16, 32),
])
def test_workspace(lib, rows, cols, dt, parts):
    d = binding.NormDesc(rows, cols, 0, dt, F32, 0, 1e-5)
    assert lib.halo_layer_norm_bwd_workspace_bytes(ctypes.byref(d)) == 2 * parts * -(-cols // 4) * 4 * 4


@pytest.mark.parametrize("rows,cols,dt,parts", [
    (432, 8192, F32, 1), (433, 8192, F32, 256), (512, 8192, F32, 256), (432, 4097, F32, 1), (512, 4097, F32, 256), (512, 4096, F32, 1),
    (512, 8193, F32, 1), (512, 4097, BF16, 1), (512, 8192, BF16, 1),
])
def test_one_launch_where_it_is_the_faster_way(lib, rows, cols, dt, parts):
    """fp32 rows of 16 to 32 KB: two launches from some 430 rows on (512 x 8192 20.6 us, one launch 22.3)."""
    test_workspace(lib, rows, cols, dt, parts)
