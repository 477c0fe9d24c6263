"""CPU: pools without in-features or without out-features, for which the C ABI does nothing: it says so and needs no workspace."""
import ctypes
import os

import pytest

from paper_2501_02625_amd import _build, binding


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_build.LIB_PATH):
        _build.build()
    return binding.load_library()


@pytest.mark.parametrize("b", [0, 1, 16, 4096])
@pytest.mark.parametrize("m,n", [(64, 0), (0, 64), (0, 0)])
@pytest.mark.parametrize("p", [0.0, 0.5])
def test_no_width_no_workspace(lib, b, m, n, p):
    d = binding.AdaptersDesc(b, m, n, 4, 16, 0, 0, p, 1, 2)
    assert lib.halo_adapters_fwd_workspace_bytes(ctypes.byref(d)) == 0
    assert lib.halo_adapters_bwd_workspace_bytes(ctypes.byref(d)) == 0
    at = ctypes.c_void_p(0x10000)
    assert lib.halo_adapters_fwd(ctypes.byref(d), at, m, at, at, None, None, at, None, 0, at, n, at, None, 0, None) == binding.HALO_OK
    assert lib.halo_adapters_bwd(ctypes.byref(d), at, n, at, m, at, at, at, None, None, at, None, 0, at, m, at, at, None, 0,
                                 None) == binding.HALO_OK
