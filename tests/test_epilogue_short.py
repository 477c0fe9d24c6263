"""Products with an epilogue and a short K: by the rule in csrc/gemm_plan.h some go to tiles of 128 x 128 (on the CPU); results of these, and of
the tiles of 256 x 128 and of two widths next to them (on the GPU)."""
import shutil
import subprocess

import pytest
import torch

from paper_2501_02625_amd import _build, binding
from tests.around_util import host, matrix, target

SHORT = [(4531, 5520, 256), (2524, 8200, 400), (5970, 4091, 768)]
OTHERS = [(2048, 4096, 512), (4531, 5520, 832), (4096, 4096, 400)]               # 256 x 128, two widths, 256 x 256

PROGRAM = r"""
#include <cstdio>
#include "gemm_plan.h"
int main() {
    long M, N, K;
    while (std::scanf("%ld %ld %ld", &M, &N, &K) == 3) {
        halo::GemmArgs a{};
        a.transB = 1; a.M = M; a.N = N; a.K = K; a.C = &a; a.config = -1;
        std::printf("%d/%d/%d\n", (int)halo::short_k_tiles128(a), halo::two_widths(a) >= 0 ? 1 : 0, halo::choose_config(a, nullptr));
    }
}
"""


def test_rule(tmp_path):
    (tmp_path / "plan.cpp").write_text(PROGRAM)
    subprocess.run([shutil.which("g++") or "g++", "-std=c++17", "-O1", "-I" + _build.INCLUDE, "-I" + _build.CSRC, str(tmp_path / "plan.cpp"), "-o",
                    str(tmp_path / "plan")], check=True)
    text = "\n".join("%d %d %d" % s for s in SHORT + OTHERS)
    said = subprocess.run([str(tmp_path / "plan")], input=text, capture_output=True, text=True, check=True).stdout.split()
    assert [s[0] for s in said] == ["1"] * len(SHORT) + ["0"] * len(OTHERS)
    assert said[len(SHORT):] == ["0/0/2", "0/1/0", "0/0/0"]


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", SHORT + OTHERS)
def test_product(M, N, K):
    from tests.gpu_util import DEV, to_dev
    from tests.test_gpu_epilogue import check, operands

    A, B, rs, cs, rng = operands(M, N, K, M + N)
    bias = torch.tensor(0.3 * rng.normal(size=N), dtype=torch.float32, device=DEV)
    res = matrix(rng.normal(size=(M, N)), torch.bfloat16, extra=1)
    (out, untouched), (zout, z_untouched) = target(M, N, torch.bfloat16), target(M, N, torch.bfloat16, extra=2)
    C, Z = binding.halo_gemm_i8_epilogue(to_dev(A), to_dev(B), row_scale=to_dev(rs), col_scale=to_dev(cs), bias=bias, activation="silu",
                                         residual=res, out=out, Z=zout)
    assert untouched() and z_untouched()
    check(A, B, rs, cs, host(bias), "silu", host(res), C, Z, torch.bfloat16, "%d x %d x %d" % (M, N, K))
