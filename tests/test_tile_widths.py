"""Which widths the planners may give a tensor-core tile (no GPU: the rule is plain C++)."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1910_04732_b200", "csrc")


@pytest.fixture(scope="module")
def allowed(tmp_path_factory):
    d = tmp_path_factory.mktemp("widths")
    src = d / "widths.cpp"
    src.write_text('#include "tile_widths.cuh"\n#include <cstdio>\n'
                   "int main() {\n  for (int bn = 0; bn <= 512; bn += 8)\n    for (int m = 0; m < 8; ++m)\n"
                   '      if (flop::tc::tile_width_ok(bn, m & 1, m & 2, m & 4)) printf("%d %d %d %d\\n", bn, m & 1, (m >> 1) & 1, m >> 2);\n}\n')
    exe = str(d / "widths")
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-I", CSRC, "-x", "c++", str(src), "-o", exe], check=True)
    return {tuple(map(int, line.split())) for line in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.splitlines()}


def test_8_bit_tiles_are_whole_64_column_groups(allowed):
    """kind::i8 has pairs of N = 32, 64, ... 256 and single CTAs of N = 8, 16, 24, 32, 48, ... 256; the epilogue stores 64 columns at a time."""
    for pair in (0, 1):
        assert {bn for bn, p, mn, b in allowed if b and not mn and p == pair} == {64, 128, 192, 256}


def test_bf16_tiles(allowed):
    assert {bn for bn, p, mn, b in allowed if not b and not mn and p} == {64, 128, 192, 208, 256}
    assert {bn for bn, p, mn, b in allowed if not b and not p} == {64, 128, 192, 256}
    assert {bn for bn, p, mn, b in allowed if not b and mn and p} == {128, 256}          # halves of whole 64-wide boxes
