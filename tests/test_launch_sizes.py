"""Launches whose threads would not fit 32 bits are made in parts or turned away on the host.  No GPU."""
import os
import subprocess

import pytest

from paper_1901_01544_amd import iwp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
AT = 0x10000                                              # never dereferenced

PROGRAM = r"""
#include <cstdio>
#include "iwp_launch_rows.hpp"
int main() {
    unsigned rows, per, across, threads;
    while (scanf("%u %u %u %u", &rows, &per, &across, &threads) == 4) {
        const int rc = iwp::in_launches(rows, per, across, threads, [&](uint32_t first, uint32_t blocks) { printf("%u %u ", first, blocks); return 0; });
        printf("%d\n", rc);
    }
    return iwp::in_launches(5, 1, 1, 1, [](uint32_t, uint32_t) { return 7; }) == 7 ? 0 : 1;
}
"""
# rows, rows of a workgroup, workgroups across a row, threads: the passes over logits, over operands and over the hidden states' gradient
CASES = [(0, 1, 1, 256), (1, 1, 1, 256), (37, 32, 1, 256), (8192, 1, 32, 256), (1 << 19, 1, 32, 256), ((1 << 19) - 1, 1, 32, 256), (1 << 20, 1, 1024, 256),
         (1 << 22, 4, 32, 256), ((1 << 22) - 3, 4, 32, 256), (1 << 20, 1, 64, 256), (1 << 20, 256, 1, 256)]


def test_rows_in_launches(tmp_path):
    source, program = tmp_path / "rows.cpp", tmp_path / "rows"
    source.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_1901_01544_amd", "csrc"), "-o", str(program), str(source)], check=True)
    out = subprocess.run([str(program)], input="".join("%d %d %d %d\n" % c for c in CASES), capture_output=True, text=True, check=True).stdout.splitlines()
    assert len(out) == len(CASES)
    parts = []
    for (rows, per, across, threads), line in zip(CASES, out):
        *numbers, rc = map(int, line.split())
        assert rc == 0
        at = 0
        for first, blocks in zip(numbers[::2], numbers[1::2]):
            assert first == at and blocks % across == 0 and 0 < blocks * threads < 1 << 32
            at = first + blocks // across * per
        assert rows <= at < rows + per
        parts.append(len(numbers) // 2)
    assert parts[:4] == [0, 1, 1, 1] and parts[4] == 2 and max(parts) > 2


@pytest.mark.parametrize("tokens,vocab,piece,fits", [(1 << 20, 1 << 22, 0, False), (1 << 20, 1 << 18, 0, True), ((1 << 18) + 1, 1 << 20, 0, False),
                                                     (1 << 18, 1 << 20, 0, True), (1 << 20, 1 << 22, 1 << 18, True), (1 << 20, 1 << 22, (1 << 18) + 1, False)])
def test_more_logits_than_a_launch_takes(tokens, vocab, piece, fits):
    """Both head calls and the workspace's size turn away the same sizes."""
    L = iwp.load()
    size = L.iwp_head_workspace_bytes(tokens, 8, vocab, 1, AT, 8, 0, piece)
    assert (size > 0) == fits
    want = iwp.IWP_EWORKSPACE if fits else iwp.IWP_EINVAL
    assert iwp._hot().iwp_head_cross_entropy(AT, 8, AT, 8, tokens, 8, vocab, 1, AT, None, 1.0, piece, AT, AT, 8, AT, 8, 1, AT, 1000, None) == want
    assert iwp._hot().iwp_head_distill(AT, 8, AT, 8, tokens, 8, vocab, 1, AT, AT, 4, 1.0, 1.0, None, 0.0, None, 1.0, piece, AT, AT, 8, AT, 8, 1, AT, 1000,
                                       None) == want
