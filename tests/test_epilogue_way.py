"""CPU test of which kernels of the product with an epilogue the shapes of its GPU tests reach, by the function that the launcher asks
(csrc/gemm_plan.h)."""
import shutil
import subprocess

import pytest
import torch

from paper_2501_02625_amd import _build
from tests import test_epilogue_long, test_epilogue_short, test_gpu_epilogue, test_gpu_epilogue_residual

BF, F32 = torch.bfloat16, torch.float32
PROGRAM = r"""
#include <cstdio>
#include "gemm_plan.h"
// each line: M, N, K, fp32 out
int main() {
    long M, N, K, f32;
    while (std::scanf("%ld %ld %ld %ld", &M, &N, &K, &f32) == 4) {
        halo::GemmArgs a{};
        a.lda = a.ldb = K; a.transB = 1; a.M = M; a.N = N; a.K = K; a.C = &a; a.c_is_f32 = (int)f32; a.ldc = N; a.config = -1;
        const halo::EpilogueWay way = halo::epilogue_way(a);
        if (way.wide >= 0) std::printf("%s\n", way.wide ? "256+192" : "192");
        else if (way.config == halo::kSmall32) std::printf("%dx%d\n", M <= 16 ? 16 : 32, (int)halo::small_tile_columns(a));
        else std::printf("%s\n", way.config == halo::kSmall64 ? "64x64" : way.config == halo::kTiles128 ? "128"
                                 : way.config == halo::kTiles256x128 ? "256x128" : "256");
    }
}
"""
ALL = {"16x16", "16x32", "16x64", "32x16", "32x32", "32x64", "64x64", "128", "256x128", "256", "192", "256+192"}


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("way")
    (d / "way.cpp").write_text(PROGRAM)
    subprocess.run([shutil.which("g++") or "g++", "-std=c++17", "-O1", "-I" + _build.INCLUDE, "-I" + _build.CSRC, str(d / "way.cpp"), "-o",
                    str(d / "way")], check=True)

    def answers(shapes):
        text = "\n".join("%d %d %d %d" % (s[0], s[1], s[2], s[3] == F32) for s in shapes)
        return subprocess.run([str(d / "way")], input=text, capture_output=True, text=True, check=True).stdout.split()

    return answers


def test_every_kernel_is_reached(ask):
    """By a GPU test that compares with 64 bits, in both types of the result."""
    for dtype in (BF, F32):
        shapes = [s + (dtype,) for s in test_gpu_epilogue.SHAPES + test_epilogue_long.SHAPES]
        shapes += [s for s in test_gpu_epilogue.TWO_WIDTHS + test_gpu_epilogue_residual.WIDE if s[3] == dtype]
        if dtype == BF:
            shapes += [s + (dtype,) for s in test_epilogue_short.SHORT + test_epilogue_short.OTHERS]
        # in fp32 these two by their number alone: test_gpu_epilogue.test_every_tile
        assert set(ask(shapes)) == ALL - ({"256", "256x128"} if dtype == F32 else set()), dtype


def test_two_widths(ask):
    """Of the four shapes of test_gpu_epilogue.TWO_WIDTHS the second goes to tiles of 128 x 128, its K is short; those here do not."""
    assert ask(test_gpu_epilogue.TWO_WIDTHS) == ["192", "128", "192", "256+192"]
    assert ask(test_gpu_epilogue_residual.WIDE) == ["192", "256+192", "256+192"]


def test_order_of_the_rules(ask):
    """Long K, short K and their neighbours (of the long ones' two have no more 64 x 64 tiles than there are compute units)."""
    assert ask([s + (BF,) for s in test_epilogue_long.SHAPES]) == ["64x64"] * 3
    assert ask([s + (BF,) for s in test_epilogue_long.NOT]) == ["128", "128", "64x64", "128", "64x64", "128"]
    assert ask([s + (BF,) for s in test_epilogue_short.SHORT + test_epilogue_short.OTHERS]) == ["128"] * 3 + ["256x128", "256+192", "256"]
