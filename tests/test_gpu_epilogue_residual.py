"""The sum of an activation and a residual that nearly cancels it: what is left is small, and as exact as the fp32 arithmetic in front of the
one rounding, in every kernel of the product with an epilogue."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import around_oracle as orc
from paper_2501_02625_amd import binding
from tests.around_util import DTYPES, HALF, U, act_bound, host, matrix, target, within
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu
# tiles of 256 x 192, and behind tiles of 256 x 256
WIDE = [(2199, 5312, 1024, torch.bfloat16), (4531, 5520, 1024, torch.bfloat16), (4231, 6688, 1024, torch.float32)]
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def call(M, N, K, act, dtype, config=-1):
    """Codes of 0: z is the bias, without any rounding.  The residual is the negative activation, rounded to dtype, times one of some factors next
    to 1."""
    rng = np.random.default_rng(M + N)
    bias = torch.tensor(rng.uniform(-4, 4, N), dtype=torch.float32, device=DEV)
    z = np.broadcast_to(host(bias), (M, N))
    a = orc.act(z, act)
    res = matrix(-a * (1 + rng.integers(-2, 3, (M, 1)) * 2.0 ** -10), dtype)
    codes = lambda rows: torch.zeros(rows, K, dtype=torch.int8, device=DEV)
    out, untouched = target(M, N, dtype)
    g = binding.gemm_desc(codes(M), codes(N), trans_b=True, out=out, config=config)
    e = binding.Epilogue(bias.data_ptr(), 1, ACTS.index(act), res.data_ptr(), res.stride(0), None, 0)
    st = binding.load_library().halo_gemm_i8_epilogue(ctypes.byref(g), ctypes.byref(e), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert st == binding.HALO_OK
    torch.cuda.synchronize()
    assert untouched()
    y = a + host(res)
    # the activation in fp32, the sum, and the one rounding (1e-40: below bf16's and fp32's smallest normal numbers steps are absolute)
    within(out, y, act_bound(z, a, act) + 2 * U * np.abs(y) + HALF[dtype] * np.abs(y) * (1 + 1e-6) + 1e-40, "%s %d x %d x %d" % (act, M, N, K))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,N,K", [(1, 4096, 64), (30, 1003, 32), (200, 1000, 64), (700, 1003, 128), (30, 77, 0)])
def test_every_activation(M, N, K, act, dtype):
    """The small kernels, tiles of 128 x 128, and the kernel of one thread an element (K = 0)."""
    call(M, N, K, act, dtype)


@pytest.mark.parametrize("config", list(binding.HALO_GEMM_CONFIGS.values()))
@pytest.mark.parametrize("dtype", DTYPES)
def test_every_tile(dtype, config):
    call(515, 700, 256, "gelu", dtype, config)


@pytest.mark.parametrize("M,N,K,dtype", WIDE)
def test_two_widths(M, N, K, dtype):
    call(M, N, K, "gelu", dtype)
