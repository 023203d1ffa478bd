"""Reads of whole 16-byte groups stay in the allocation, also for the last columns of a wider matrix."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2501_01951_amd", "csrc")


@pytest.fixture(scope="module")
def second_group(tmp_path_factory):
    """The rule of the kernels, as a table [cols][col / 4]."""
    d = tmp_path_factory.mktemp("rules")
    (d / "t.cpp").write_text('#include <cstdio>\n#include "load_rules.h"\n'
                             'int main() { for (int n = 1; n <= 64; ++n) { for (int c = 0; c < n; c += 4)'
                             ' std::printf("%d ", mixgcn::second_group(c, n)); std::printf("\\n"); } }\n')
    subprocess.run(["g++", "-std=c++17", "-I", CSRC, "-o", str(d / "t"), str(d / "t.cpp")], check=True, timeout=60)
    out = subprocess.run([str(d / "t")], check=True, capture_output=True, text=True, timeout=60).stdout
    table = [[int(v) for v in line.split()] for line in out.splitlines()]
    return lambda col, cols, pitch: table[cols - 1][col // 4]


def reads_past_the_end(rule):
    """Slices [:, first:first + cols] of two rows on a pitch of whole groups whose last element is read by the rule."""
    bad = []
    for pitch in range(4, 65, 4):
        for first in range(0, pitch, 4):
            for cols in range(1, pitch - first + 1):
                for col in range(0, cols, 4):
                    last = pitch + first + max(col, rule(col, cols, pitch)) + 3
                    if last >= 2 * pitch:
                        bad.append((pitch, first, cols, col))
    return bad


def test_second_group_of_a_row(second_group):
    assert reads_past_the_end(second_group) == []
    for cols in range(1, 65):
        for col in range(0, cols, 4):
            assert second_group(col, cols, 0) == (col + 4 if col + 4 < cols else col)


def test_the_check_finds_a_rule_that_goes_by_the_pitch():
    assert reads_past_the_end(lambda col, cols, pitch: col) == []
    assert (64, 60, 4, 0) in reads_past_the_end(lambda col, cols, pitch: col + 4 if col + 4 < pitch else col)
