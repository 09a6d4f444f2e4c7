"""Which kernels the gated projections run in where only h is wanted.  CPU only: the rule is host
code."""
import os
import subprocess

import pytest

from expert_tiles import CSRC, ROOT

PROGRAM = """
#include <stdio.h>
#include "groups.h"
// rows groups(0: one without offsets) hidden others -> with the products, h alone
int main() {
  int rows, groups, hidden, others;
  static const int32_t kOffsets = 0;
  while (scanf("%d %d %d %d", &rows, &groups, &hidden, &others) == 4) {
    const gnmr::GroupArgs g{groups == 0 ? nullptr : &kOffsets, nullptr, groups == 0 ? 1 : groups, 1,
                            rows};
    printf("%d %d\\n", gnmr::gated_linear_streams(g, hidden, others, true),
           gnmr::gated_linear_streams(g, hidden, others, false));
  }
}
"""

# rows, groups, hidden, the other features; one after the other with the products, and h alone
SHAPES = {
    (8192, 0, 11008, 4096): (1, 0),
    (8192, 0, 13824, 5120): (1, 0),
    (4096, 0, 4096, 4096): (1, 0),
    (32768, 16, 1408, 2048): (1, 0),
    (24576, 32, 1408, 2048): (1, 1),
    (24640, 64, 1408, 2048): (1, 1),
    (1024, 0, 11008, 4096): (1, 1),
    (64, 0, 11008, 4096): (0, 0),
    (8192, 8, 2000, 2056): (0, 0),
}


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    from paper_2606_00539_amd import _build as B

    at = tmp_path_factory.mktemp("alone")
    (at / "alone.hip").write_text(PROGRAM)
    flags = [f for f in B.HIPCC_FLAGS if f not in ("-shared", "-O3")]
    subprocess.run([B.hipcc(), *flags, "-O1", "-I", CSRC, "-I", os.path.join(ROOT, "include"), "-o",
                    str(at / "alone"), str(at / "alone.hip")], check=True, capture_output=True)
    return at / "alone"


def test_h_alone_of_large_groups_runs_in_tiles(rule):
    text = "".join("%d %d %d %d\n" % s for s in SHAPES)
    out = subprocess.run([str(rule)], input=text, check=True, capture_output=True, text=True,
                         timeout=60).stdout.split("\n")[:-1]
    assert [(s, o) for s, o in zip(SHAPES, out) if o != "%d %d" % SHAPES[s]] == []
