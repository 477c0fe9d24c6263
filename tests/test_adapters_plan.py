"""CPU test of which way the rules in csrc/adapters_plan.h send the shapes of the GPU tests: a test that is there for one kernel keeps
reaching it when a rule changes, or fails here."""
import shutil
import subprocess

import pytest

from paper_2501_02625_amd import _build
from tests import test_gpu_adapters_tall as tall

PROGRAM = r"""
#include <cstdio>
#include "adapters_plan.h"
// each line: tokens, columns, what the pool allots to an adapter
int main() {
    long b, wide, rank;
    while (std::scanf("%ld %ld %ld", &b, &wide, &rank) == 3) std::printf("%d\n", halo::adapters::wide_tile_tokens(b, wide, (int)rank));
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(PROGRAM)
    subprocess.run([shutil.which("g++") or "g++", "-std=c++17", "-O1", "-I" + _build.CSRC, str(d / "plan.cpp"), "-o", str(d / "plan")],
                   check=True)

    def answers(lines):
        text = "\n".join(" ".join(map(str, l)) for l in lines)
        return [int(x) for x in subprocess.run([str(d / "plan")], input=text, capture_output=True, text=True, check=True).stdout.split()]

    return answers


def test_shapes_of_the_tests_of_tall_tiles(ask):
    assert ask((b, wide, rank) for rank, b, wide, tile in tall.SHAPES) == [tile for *_, tile in tall.SHAPES]


def test_every_template_is_reached(ask):
    """The ranks' four templates, each with every tile that the rule has for it."""
    template = lambda rank: 0 if rank <= 16 else 1 if rank <= 32 else 2 if rank <= 64 else 4
    reached = {(template(rank), tile) for rank, _, _, tile in tall.SHAPES}
    assert reached == {(t, tile) for t in (0, 1, 2) for tile in (64, 256)} | {(4, 128)}


def test_tiles_of_any_size(ask):
    """What the rule can answer, and that taller tiles come with more tokens and columns."""
    sizes = [(b, wide) for b in (1, 63, 64, 65, 257, 1000, 2048, 4097, 1 << 16, 1 << 22) for wide in (8, 512, 520, 4096, 14336, 1 << 20)]
    for rank, tiles in ((8, {16, 64, 256}), (64, {16, 64, 256}), (72, {16, 128}), (128, {16, 128})):
        said = dict(zip(sizes, ask((b, wide, rank) for b, wide in sizes)))
        assert set(said.values()) == tiles
        for wide in {w for _, w in sizes}:
            of_b = [said[s] for s in sorted(sizes) if s[1] == wide]
            assert of_b == sorted(of_b)
