"""Warps to a row of the log-probabilities (csrc/policy_plan.h), on the CPU: the number that leaves fewer
places unused in the turns that an SM's rows take."""
import subprocess
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent
PROGRAM = r'''
#include <stdio.h>
#include "policy_plan.h"
int main(void) {
    long long rows;
    int sm, r4, r8;
    while (scanf("%lld %d %d %d", &rows, &sm, &r4, &r8) == 4) printf("%d\n", adama::warps_to_a_row(rows, sm, r4, r8));
    return 0;
}
'''


@pytest.fixture(scope="module")
def warps(tmp_path_factory):
    d = tmp_path_factory.mktemp("warps")
    (d / "warps.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", str(ROOT / "paper_2305_19982_b200" / "csrc"),
                    str(d / "warps.cpp"), "-o", str(d / "warps")], check=True)

    def ask(rows, r4, r8, sm=148):
        text = "".join(f"{t} {sm} {r4} {r8}\n" for t in rows)
        out = subprocess.run([str(d / "warps")], input=text, capture_output=True, text=True, check=True).stdout.split()
        return [int(x) for x in out]

    return ask


def test_the_faster_number_where_they_differ_by_more_than_a_tenth(warps):
    """Rows per SM against measured times of fp32 rows of 128256 (10 and 5 resident): 740 rows 65.6 us with
    4 warps and 57.4 with 8, 800 68.2 and 78.5, 1600 150.9 and 133.2, 2048 166.3 and 151.3."""
    assert warps([740, 800, 1600, 2048], 10, 5) == [8, 4, 8, 8]


def test_whole_turns_of_the_smaller_ones_stay_with_them(warps):
    for r4, r8 in [(10, 5), (12, 6), (16, 8)]:
        assert warps([148 * r4, 148 * 2 * r4, 148 * r8, 148 * r8 + 1, 148 * r4 + 1], r4, r8) == [4, 4, 8, 4, 8]
        assert warps([148 * 2 * r4 + 1, 148 * 5 * r4, 10 ** 9], r4, r8) == [4, 4, 4]       # many turns
    assert warps([1, 147, 148, 149], 10, 5) == [8, 8, 8, 8]                                # one turn of either


def test_residencies_without_a_common_measure(warps):
    assert warps([148 * 6, 148 * 8], 7, 3) == [8, 8] and warps([148 * 3, 148 * 7], 7, 3) == [8, 4]
    assert warps([5], 1, 1, sm=1) == [4]
