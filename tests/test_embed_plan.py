"""What the gradient of the lookup decides from sizes and tokens alone (csrc/embed_plan.h), on the host."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2001_00532_amd", "csrc")
CXX = shutil.which("g++")

pytestmark = pytest.mark.skipif(CXX is None, reason="no host compiler")


def compiled(tmp_path, body, run=True):
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text('#include "embed_plan.h"\n#include <cstdio>\nusing namespace psk;\n' + body)
    r = subprocess.run([CXX, "-std=c++17", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout if run else ""


def test_places_of_any_token(tmp_path):
    """A constant expression must not overflow: these do not compile where the difference is one of signed numbers."""
    tokens = ["-2147483647 - 1", "-2147483647", "-1", "0", "4", "5", "6", "14", "15", "268435200", "2147483647"]
    value = [-2 ** 31, -2 ** 31 + 1, -1, 0, 4, 5, 6, 14, 15, 268435200, 2 ** 31 - 1]
    checks = ["static_assert((place_from(%s, %d) < %du) == %s);" % (t, first, count, "true" if first <= v < first + count else "false")
              for first, count in ((0, 1), (5, 10), (512, 512), (2 ** 28 - 257, 1), (2 ** 28 - 768, 512)) for t, v in zip(tokens, value)]
    compiled(tmp_path, "\n".join(checks) + "\nint main() {}\n")


def test_every_way_is_tested(tmp_path):
    """The GPU tests' sizes: where each is sorted, how many columns a wave has, how many positions a tile."""
    pytest.importorskip("torch")
    from test_gpu_embed_ways import DIGITS, RANGES, SCANNED

    def plan(sizes):
        calls = "".join('std::printf("%%d %%d %%d %%d\\n", (int)way_of(%d, %d, %d, 4), quads_per_lane(%d), tile_of(%d, %d), %d);\n' % (n, rows, dim, dim, n, dim, dim) for n, rows, dim in sizes)
        names = 'std::printf("%d %d %d\\n", BY_RANGES, BY_DIGITS, BY_SCANNED_DIGITS);\n'
        lines = [tuple(map(int, line.split())) for line in compiled(tmp_path, "int main() {\n" + names + calls + "}\n").splitlines()]
        return lines[0], lines[1:]
    (ranges, digits, scanned), got = plan(RANGES + DIGITS + SCANNED)
    assert [g[0] for g in got] == [ranges] * len(RANGES) + [digits] * len(DIGITS) + [scanned] * len(SCANNED)
    # quads per lane, and whether several waves share a row
    assert {(j, dim > 256 * j) for _, j, _, dim in got[:len(RANGES)]} >= {(1, False), (2, False), (2, True), (3, False), (3, True)}
    assert {tile for _, _, tile, _ in got} == {8, 16, 32, 64} and any(j == 2 and tile == 64 for _, j, tile, _ in got)
    assert (262144, 262145) == (max(n for n, _, _ in DIGITS), min(n for n, _, _ in SCANNED))


def test_a_workspace_has_room_for_fewer_tokens(tmp_path):
    """most_tiles(n, dim) against the tiles of every smaller number of tokens."""
    body = """
int main()
{
    for (int64_t dim : {1, 3, 4, 64, 255, 256, 257, 300, 512, 513, 768, 769, 1024, 1025, 2048, 4099, 9000, 70000, 1 << 20, 1 << 28}) {
        int64_t most = 0;
        for (int64_t n = 1; n <= 40000; ++n) {
            most = std::max(most, (n + tile_of(n, dim) - 1) / tile_of(n, dim));
            if (most > most_tiles(n, dim)) std::printf("%lld %lld\\n", (long long)n, (long long)dim);
        }
        for (int64_t n = 40000; n <= 1 << 24; n += 97) {
            most = std::max(most, (n + tile_of(n, dim) - 1) / tile_of(n, dim));
            if (most > most_tiles(n, dim)) std::printf("%lld %lld\\n", (long long)n, (long long)dim);
        }
    }
}
"""
    assert compiled(tmp_path, body) == ""
