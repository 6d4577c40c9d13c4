"""How products of 8-bit integers are cut up (csrc/gemm_i8_plan.h), on the host: the sizes that the GPU tests run reach every shape of tile."""
import os
import shutil
import subprocess

import pytest

pytest.importorskip("torch")
from test_gpu_i8_shapes import PARTS, WHOLE  # noqa: E402

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2001_00532_amd", "csrc")
CXX = shutil.which("g++")

pytestmark = pytest.mark.skipif(CXX is None, reason="no host compiler")

SOURCE = """
#include "gemm_i8_plan.h"
#include <cstdio>
using namespace psk;
int main()
{
    for (const Shape &s : SHAPES) std::printf("%d %d\\n", s.tokens, s.channels);
    std::printf("\\n");
    for (int r, c, n; std::scanf("%d %d %d", &r, &c, &n) == 3;) {
        const Choice k = choose(r, c, n);
        std::printf("%d %d %d\\n", k.shape, k.parts, k.part_cols);
    }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    """(shapes, a function from sizes to (shape, parts, columns of a part))."""
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(SOURCE)
    r = subprocess.run([CXX, "-std=c++17", "-Wall", "-Werror", "-I", CSRC, str(d / "plan.cpp"), "-o", str(d / "plan")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def ask(sizes):
        out = subprocess.run([str(d / "plan")], input="".join("%d %d %d\n" % s for s in sizes), capture_output=True, text=True, check=True).stdout
        first, rest = out.split("\n\n")
        return [tuple(map(int, line.split())) for line in first.splitlines()], [tuple(map(int, line.split())) for line in rest.splitlines()]
    return ask


# of the instances in gemm_i8.hip
STAGES = {(16, 16): 8, (16, 32): 8, (32, 32): 6, (32, 64): 4, (64, 32): 4, (64, 64): 4, (128, 64): 4, (128, 128): 4, (256, 128): 3, (256, 256): 2}


@pytest.mark.parametrize("what", ["whole", "parts"])
def test_every_shape_is_tested(plan, what):
    sizes = WHOLE if what == "whole" else PARTS
    shapes, chosen = plan(sizes)
    assert set(shapes) == set(STAGES)
    met = set()
    for (rows, cols, n), (k, parts, part_cols) in zip(sizes, chosen):
        tokens, channels = shapes[k]
        assert (parts > 1) == (what == "parts") and cols % 16 and cols % 128 and n % tokens and rows % channels, (rows, cols, n)
        assert ((cols if parts == 1 else part_cols) + 127) // 128 > STAGES[shapes[k]], (rows, cols, n)
        met.add(shapes[k])
    assert met == set(shapes) - ({(256, 256)} if what == "parts" else set()), set(shapes) - met


def test_parts_fit_their_room(plan):
    """The sums of all parts fit the workspace, every part has columns, and the largest tiles are never chosen for parts."""
    sizes = [(rows, cols, n) for cols in (1, 127, 128, 129, 1000, 2049, 4097, 9000, 16384, 33000, 131071) for n in (1, 5, 16, 17, 33, 70, 130, 260, 1000, 2100, 4200, 9000, 40000)
             for rows in (1, 4, 9, 17, 33, 70, 130, 260, 1000, 2100, 5000, 20000, 100000)]
    shapes, chosen = plan(sizes)
    for (rows, cols, n), (k, parts, part_cols) in zip(sizes, chosen):
        if parts > 1:
            assert parts * n * ((rows + 3) // 4 * 4) * 4 <= 16 << 20 and cols > 128 and shapes[k] != (256, 256), (rows, cols, n)
            assert part_cols % 128 == 0 and part_cols * (parts - 1) < cols <= part_cols * parts, (rows, cols, n)
