"""Row numbers of the recurrence at the largest batches that it accepts, on the host."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1809_00832_amd", "csrc")

PROGRAM = r"""
#include <cstdio>
#include "recur_rows.hpp"

int main()
{
    int tail, slot, wave, slots;
    while (std::scanf("%d %d %d %d", &tail, &slot, &wave, &slots) == 4) std::printf("%lld\n", tl::rec_behind(tail, slot, wave, slots));
}
"""


def test_rows_behind_the_last_sentence_pass_32_bits(tmp_path):
    """tail + slot is 2^31 and more from 2^16 sentences on where nearly 2^31 rows are in use: no row of the batch, and none in front of it."""
    most = 2 ** 31 - 2 ** 16 - 1
    cases = [(0, 0, 0, 1), (5, 3, 2, 7), (most, 2 ** 16 - 1, 0, 2 ** 17), (most, 2 ** 16 + 1, 0, 2 ** 17), (most, 2 ** 22 - 2, 3, 2 ** 22 - 1), (2 ** 30, 2 ** 22 - 2, 7, 2 ** 22 - 1)]
    source, program = tmp_path / "rows.cpp", tmp_path / "rows"
    source.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC, "-o", str(program), str(source)], check=True)
    got = subprocess.run([str(program)], input="\n".join("%d %d %d %d" % c for c in cases), capture_output=True, text=True, check=True).stdout.split()
    assert [int(v) for v in got] == [tail + slot + wave * slots for tail, slot, wave, slots in cases]
