"""Shapes of the gated products by the kernels that they run in.  test_block_tiles.py checks on the
CPU that each still does, test_gpu_gated.py runs them."""
import os
import subprocess

from expert_tiles import CSRC, ROOT, loads

PROGRAM = """
#include <stdio.h>
#include <string.h>
#include "groups.h"
// op rows groups(0: one without offsets) hidden others -> what runs
int main() {
  char op[16];
  int rows, groups, hidden, others;
  static const int32_t kOffsets = 0;
  while (scanf("%15s %d %d %d %d", op, &rows, &groups, &hidden, &others) == 5) {
    const gnmr::GroupArgs g{groups == 0 ? nullptr : &kOffsets, nullptr, groups == 0 ? 1 : groups, 1,
                            rows};
    if (!strcmp(op, "linear") ? gnmr::gated_linear_streams(g, hidden, others, true)
                              : gnmr::gated_dgrad_streams(g, hidden, others)) {
      puts("stream");
      continue;
    }
    const gnmr::RowLaunch r = !strcmp(op, "linear") ? gnmr::row_launch(g, 2 * hidden, others, 2)
                                                    : gnmr::row_launch(
                                                          g, hidden, others, 2,
                                                          gnmr::kGatedDgradBeside);
    printf("%d %s%s\\n", r.tile, r.split ? "rounds and rest" : "all",
           !strcmp(op, "linear") && r.tile == 64 && gnmr::gated_weights_once(g) ? " once" : "");
  }
}
"""


def build(folder):
    """The program that tells what runs, compiled in `folder`: cases -> ["edge launches"]."""
    from paper_2606_00539_amd import _build as B

    (folder / "gated.hip").write_text(PROGRAM)
    flags = [f for f in B.HIPCC_FLAGS if f not in ("-shared", "-O3")]
    subprocess.run([B.hipcc(), *flags, "-O1", "-I", CSRC, "-I", os.path.join(ROOT, "include"), "-o",
                    str(folder / "gated"), str(folder / "gated.hip")], check=True,
                   capture_output=True)

    def run(cases):
        text = "".join("%s %d %d %d %d\n" % c for c in cases)
        out = subprocess.run([str(folder / "gated")], input=text, check=True, capture_output=True,
                             text=True, timeout=60).stdout.split("\n")[:-1]
        assert len(out) == len(cases)
        return out
    return run


# hidden and the other features, the rows of the experts (None: one without offsets), rows of
# nobody, and what the projections (kept) and their gradient run in; but for the streams' the other
# features are no multiples of a step's 64 values
SHAPES = {
    "64 tiles, 70 experts": (88, 72, loads(70, 600, 1), 5, ("64 all once", "64 all")),
    "64 tiles, one expert": (80, 136, None, 333, ("64 all", "64 all")),
    "128 tiles, 70 experts": (488, 200, loads(70, 300, 2), 9, ("128 all", "64 all")),
    "128 tiles, 8 experts": (856, 360, loads(8, 1200, 4), 70, ("128 all", "64 all")),
    "128 tiles, one expert": (456, 712, None, 3000, ("128 all", "64 all")),
    "256 tiles, 100 experts": (608, 136, loads(100, 200, 5), 3, ("256 all", "128 all")),
    "256 tiles, 8 experts": (2880, 136, loads(8, 920, 6), 33, ("256 all", "128 all")),
    "256 tiles, one expert": (200, 136, None, 18500, ("256 all", "128 all")),
    "256 tiles of the gradient": (2000, 1000, loads(8, 4000, 7), 33, ("128 all", "256 all")),
    "256 tiles of the gradient, one expert": (2000, 520, None, 5000, ("128 all", "256 all")),
    "rounds and rest, 8 experts": (2504, 5128, loads(8, 4200, 8), 259,
                                   ("256 rounds and rest", "256 rounds and rest")),
    "rounds and rest of the gradient, one expert": (3816, 5128, None, 10115,
                                                    ("256 all", "256 rounds and rest")),
    "streams, 70 experts": (1000, 2048, loads(70, 9000, 9), 300, ("stream", "stream")),
    "streams, 4 experts": (5504, 4096, loads(4, 1000, 10), 5, ("stream", "stream")),
    "streams, one expert": (4096, 4096, None, 4093, ("stream", "stream")),
    "streams, one expert of fewer rows": (5504, 2048, None, 2041, ("stream", "stream")),
    "streams, 200 experts": (200, 256, loads(200, 25000, 12), 77, ("stream", "stream")),
    "streams of four steps": (2000, 256, None, 3001, ("stream", "stream")),
    "streams of five steps, 20 experts": (1000, 320, loads(20, 3000, 11), 40, ("stream", "stream")),
    "stream of the gradient, fewer than 256 tiles": (2752, 4096, None, 2000, ("256 all", "stream")),
    "rounds and rest, one expert": (1912, 5128, None, 10115, ("256 rounds and rest", "128 all")),
}


def shape(which, name):
    """(op, rows, groups, hidden, others) of a case, as the program takes it."""
    H, K, counts, pad, _ = SHAPES[name]
    rows = pad if counts is None else sum(counts) + pad
    return which, rows, 0 if counts is None else len(counts), H, K
