"""Products with an epilogue and a long K whose 64 x 64 tiles are more than the compute units: by the rule in csrc/gemm_plan.h they go to
the small kernel (on the CPU), and there they give what the tiled kernels give and the formulas say (on the GPU)."""
import ctypes
import shutil
import subprocess

import numpy as np
import pytest
import torch

from paper_2501_02625_amd import _build, binding
from tests.around_util import DTYPES, host, matrix, target

SHAPES = [(529, 2044, 8192), (1075, 1024, 8208), (266, 4096, 8960)]
NOT = [(529, 2044, 4096), (529, 2112, 8192), (125, 8192, 8192), (2163, 512, 8192), (500, 2048, 8192), (266, 5120, 8192)]

PROGRAM = r"""
#include <cstdio>
#include "gemm_plan.h"
int main() {
    long M, N, K;
    while (std::scanf("%ld %ld %ld", &M, &N, &K) == 3) {
        halo::GemmArgs a{};
        a.transB = 1; a.M = M; a.N = N; a.K = K; a.config = -1;
        std::printf("%d\n", (int)halo::small_tiles_twice(a));
    }
}
"""


def test_rule(tmp_path):
    (tmp_path / "plan.cpp").write_text(PROGRAM)
    subprocess.run([shutil.which("g++") or "g++", "-std=c++17", "-O1", "-I" + _build.INCLUDE, "-I" + _build.CSRC, str(tmp_path / "plan.cpp"), "-o",
                    str(tmp_path / "plan")], check=True)
    text = "\n".join("%d %d %d" % s for s in SHAPES + NOT)
    said = subprocess.run([str(tmp_path / "plan")], input=text, capture_output=True, text=True, check=True).stdout.split()
    assert said == ["1"] * len(SHAPES) + ["0"] * len(NOT)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_product(M, N, K, dtype):
    from tests.gpu_util import DEV, to_dev
    from tests.test_gpu_epilogue import check, operands

    A, B, rs, cs, rng = operands(M, N, K, M + N)
    a, b, r, c = (to_dev(v) for v in (A, B, rs, cs))
    bias = torch.tensor(0.3 * rng.normal(size=N), dtype=torch.float32, device=DEV)
    res = matrix(rng.normal(size=(M, N)), dtype, extra=1)
    (out, untouched), (zout, z_untouched) = target(M, N, dtype), target(M, N, dtype, extra=2)
    C, Z = binding.halo_gemm_i8_epilogue(a, b, row_scale=r, col_scale=c, bias=bias, activation="gelu", residual=res, out=out, Z=zout)
    assert untouched() and z_untouched()
    check(A, B, rs, cs, host(bias), "gelu", host(res), C, Z, dtype, "%d x %d x %d" % (M, N, K))
    again, z = target(M, N, dtype)[0], target(M, N, dtype)[0]
    g = binding.gemm_desc(a, b, trans_b=True, row_scale=r, col_scale=c, out=again, config=4)
    e = binding.Epilogue(bias.data_ptr(), 1, 2, res.data_ptr(), res.stride(0), z.data_ptr(), z.stride(0))
    st = binding.load_library().halo_gemm_i8_epilogue(ctypes.byref(g), ctypes.byref(e), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert st == binding.HALO_OK
    torch.cuda.synchronize()
    assert np.array_equal(host(again), host(C)) and np.array_equal(host(z), host(Z))
