"""Host-side check of the rule that picks a form for packed prompts (``tile_rules.hpp``), compiled by itself with the host
compiler: where one form was measured clearly faster for prompts of one length and for uneven ones, the rule takes it."""
import subprocess

import pytest

from paper_2607_19438_amd import build

MAIN = """
#include <cstdio>
#include "tile_rules.hpp"
int main() {
  long d64, T, R, heads;
  while (std::scanf("%ld %ld %ld %ld", &d64, &T, &R, &heads) == 4) std::printf("%d\\n", (int)qg::attn_packed_split(d64 != 0, T, R, heads));
}
"""

# head dimension, prompts, workgroups of 128 rows: time of the 64-row form over the other's, 16 heads (one length, uneven)
MEASURED = [
    (64, 1, 512, 0.80, 0.80), (64, 1, 640, 0.88, 0.88), (64, 1, 704, 0.92, 0.92), (64, 2, 512, 0.85, 0.86), (64, 2, 640, 0.78, 0.85),
    (64, 2, 704, 0.83, 0.87), (64, 3, 256, 0.84, 0.85), (64, 3, 512, 0.87, 0.83), (64, 3, 576, 0.96, 0.80), (64, 3, 640, 0.98, 0.82),
    (64, 3, 704, 0.98, 0.86), (64, 4, 448, 0.97, 0.89), (64, 5, 448, 0.84, 0.81), (64, 40, 384, 0.92, 0.85), (128, 2, 512, 0.86, 0.90),
    (128, 3, 384, 0.90, 0.86), (128, 4, 256, 0.93, 0.83), (128, 2, 896, 1.13, 1.01), (128, 3, 896, 1.04, 1.03), (128, 4, 896, 0.99, 1.05),
]


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    d = tmp_path_factory.mktemp("rule")
    (d / "main.cpp").write_text(MAIN)
    subprocess.run(["g++", "-std=c++20", "-I", build.CSRC, str(d / "main.cpp"), "-o", str(d / "rule")], check=True)
    return str(d / "rule")


@pytest.mark.parametrize("D,R,wide,even,uneven", MEASURED)
def test_the_faster_form_is_taken(rule, D, R, wide, even, uneven):
    call = f"{int(D == 64)} {wide // 16 * 128 - 17} {R} 16\n"
    split = subprocess.run([rule], input=call, capture_output=True, text=True, check=True).stdout.strip() == "1"
    assert split == ((even + uneven) / 2 < 1)
