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
