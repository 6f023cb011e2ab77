"""Which workgroup takes which tile or half of one: every tile once, nothing beyond the last.  No GPU."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include <cstdio>
#include "iwp_halves.hpp"
int main() {
    unsigned tiles, bound;
    while (scanf("%u %u", &tiles, &bound) == 2) {
        for (unsigned block = 0; block < bound + iwp::MOST_HALVES; ++block) {
            iwp::TilePart part;
            uint32_t whole;
            if (iwp::part_of(block, tiles, &part, &whole)) printf("%u:%u ", part.tile, part.half);
        }
        printf("\n");
    }
}
"""


def test_every_tile_once(tmp_path):
    source, program = tmp_path / "halves.cpp", tmp_path / "halves"
    source.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_1901_01544_amd", "csrc"), "-o", str(program), str(source)], check=True)
    cases = [(tiles, tiles + more) for tiles in (0, 1, 2, 127, 128, 129, 200, 255, 256, 257, 300, 384, 385, 511, 512, 513, 640, 641, 1100, 1168) for more in (0, 1, 300)]
    out = subprocess.run([str(program)], input="".join("%d %d\n" % c for c in cases), capture_output=True, text=True, check=True).stdout.splitlines()
    assert len(out) == len(cases)
    for (tiles, _), line in zip(cases, out):
        parts = [tuple(map(int, p.split(":"))) for p in line.split()]
        whole, upper, lower = ([t for t, h in parts if h == half] for half in range(3))
        assert sorted(whole + upper) == list(range(tiles)) and upper == lower and len(upper) <= 128
        assert (len(parts) + 255) // 256 <= max(1, (tiles + 255) // 256) if tiles else not parts      # never a round more
