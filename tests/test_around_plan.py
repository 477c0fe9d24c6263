"""CPU test of which kernels the shapes of tests/test_gpu_epilogue.py reach by the rules in csrc/gemm_plan.h: every one of them is there
for a kernel, and fails here when a rule sends it elsewhere."""
import shutil
import subprocess

import pytest
import torch

from paper_2501_02625_amd import _build
from tests import test_gpu_epilogue as gpu

PROGRAM = r"""
#include <cstdio>
#include "gemm_plan.h"
// each line: M, N, K, fp32 out
int main() {
    long M, N, K, f32;
    while (std::scanf("%ld %ld %ld %ld", &M, &N, &K, &f32) == 4) {
        halo::GemmArgs a{};
        a.lda = a.ldb = K; a.transB = 1; a.M = M; a.N = N; a.K = K; a.C = &a; a.c_is_f32 = (int)f32; a.ldc = N; a.config = -1;
        const long wide = (long)halo::two_widths(a), config = halo::choose_config(a, nullptr);
        if (wide >= 0) std::printf("%s\n", wide ? "256+192" : "192");
        else if (config == halo::kSmall32) std::printf("%dx%d\n", M <= 16 ? 16 : 32, (int)halo::small_tile_columns(a));
        else std::printf("%s\n", config == halo::kSmall64 ? "64x64" : config == halo::kTiles128 ? "128" : config == halo::kTiles256x128 ? "256x128" : "256");
    }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(PROGRAM)
    subprocess.run([shutil.which("g++") or "g++", "-std=c++17", "-O1", "-I" + _build.INCLUDE, "-I" + _build.CSRC, str(d / "plan.cpp"), "-o",
                    str(d / "plan")], check=True)

    def answers(shapes):
        text = "\n".join("%d %d %d %d" % s for s in shapes)
        return subprocess.run([str(d / "plan")], input=text, capture_output=True, text=True, check=True).stdout.split()

    return answers


def test_shapes_reach_every_small_kernel(ask):
    for f32 in (0, 1):
        said = set(ask([s + (f32,) for s in gpu.SHAPES]))
        assert {"16x16", "16x32", "16x64", "32x16", "32x32", "32x64", "64x64", "128"} <= said          # the larger tiles: test_every_tile


def test_shapes_of_two_widths(ask):
    assert ask([s[:3] + (int(s[3] == torch.float32),) for s in gpu.TWO_WIDTHS]) == ["192", "256+192", "192", "256+192"]
