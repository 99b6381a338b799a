"""Host-side checks of how a table reordering is cut into workgroups (``tile_rules.hpp``, compiled by itself with the host
compiler): every block of columns has one workgroup in each kernel, and what the workgroups read beside their own blocks
grows with the tables and not with their square. No test here touches a GPU."""
import random
import subprocess

import pytest

from paper_2607_19438_amd import build

MAIN = """
#include <cstdio>
#include "tile_rules.hpp"
int main() {
  for (long r, b; std::scanf("%ld %ld", &r, &b) == 2;) {
    const qg::ReorderSplit p = qg::reorder_split(r, b);
    std::printf("%ld %ld %ld %ld\\n", p.each, p.parts, p.release_each, p.release);
  }
}
"""


@pytest.fixture(scope="module")
def split(tmp_path_factory):
    d = tmp_path_factory.mktemp("split")
    (d / "main.cpp").write_text(MAIN)
    subprocess.run(["g++", "-std=c++20", "-Wall", "-Werror", "-I", build.CSRC, str(d / "main.cpp"), "-o", str(d / "split")], check=True)

    def run(calls):
        text = "".join(f"{r} {b}\n" for r, b in calls)
        out = subprocess.run([str(d / "split")], input=text, capture_output=True, text=True, check=True).stdout
        return [tuple(int(x) for x in line.split()) for line in out.splitlines()]
    return run


def calls():
    rng = random.Random(1)
    out = [(1, 1), (64, 1), (512, 32), (65536, 1), (65536, 128), (1, (1 << 31) // 256), (2048, 2), (2049, 2), (1024, 1), (1025, 1)]
    for _ in range(2000):
        r = int(2 ** rng.uniform(0, 16))
        out.append((r, max(1, int(2 ** rng.uniform(0, 31) / r / 256))))          # rows times columns below 2^31
    return out


def test_every_block_has_a_workgroup(split):
    for (r, b), (each, parts, release_each, release) in zip(calls(), split(calls())):
        assert each >= 1 and parts * each >= b > (parts - 1) * each
        assert release_each >= 1 and release * release_each >= r * b > (release - 1) * release_each


def test_reads_do_not_grow_with_the_square(split):
    """The second kernel's workgroups read all blocks' counts each; the first's up to 65536 rows' lengths and parents each."""
    for (r, b), (each, parts, release_each, release) in zip(calls(), split(calls())):
        assert release <= 2048 and r * parts <= max(2048, r)
        assert 4 * release * r * b <= 8 * 1024 * (r * b)          # bytes: eight times those of a row of all blocks, 1024 each
        if r * b <= 2048:                                        # few blocks: a workgroup to each
            assert each == 1 and release_each == 1
