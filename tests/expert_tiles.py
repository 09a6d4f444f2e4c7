"""Shapes of the grouped products and of the orthogonalisation's by the kernels that they run in.
test_expert_tiles.py checks on the CPU that each still does, test_gpu_expert_tiles.py runs them."""
import os
import subprocess

import numpy as np

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_00539_amd", "csrc")

PROGRAM = """
#include <stdio.h>
#include <string.h>
#include "groups.h"
// op rows groups(0: one without offsets) out in, or "batch" count m n and a 0 -> what runs
int main() {
  char op[16];
  int rows, groups, out, in;
  static const int32_t kOffsets = 0;
  while (scanf("%15s %d %d %d %d", op, &rows, &groups, &out, &in) == 5) {
    const gnmr::GroupArgs g{groups == 0 ? nullptr : &kOffsets, nullptr, groups == 0 ? 1 : groups, 1,
                            rows};
    if (!strcmp(op, "batch")) {
      for (auto what : {gnmr::BatchProduct::kOfRows, gnmr::BatchProduct::kOfSquares,
                        gnmr::BatchProduct::kOntoRows}) {
        const gnmr::BatchLaunch b =
            gnmr::batch_launch(what, rows, (groups + 63) / 64 * 64, (out + 63) / 64 * 64);
        printf(b.large == 0 ? "%s%d" : b.edge == 0 ? "%s256" : "%s256+%d",
               what == gnmr::BatchProduct::kOfRows ? "" : " ", b.edge);
      }
      puts("");
      continue;
    }
    if (!strcmp(op, "wgrad")) {
      const int edge = gnmr::wgrad_tile(g, out, in);
      const int per = (out + edge - 1) / edge * ((in + edge - 1) / edge);
      printf("%d %s\\n", edge, g.num == 1 || per < gnmr::kSharedTiles ? "whole"
                               : per % gnmr::kNumXcd == 0             ? "eighths" : "uneven eighths");
      continue;
    }
    const bool dgrad = !strcmp(op, "dgrad"), codes = !strcmp(op, "quantized");
    const gnmr::RowLaunch r = gnmr::row_launch(g, dgrad ? in : out, dgrad ? out : in, codes ? 1 : 2);
    printf("%d %s\\n", r.tile, r.split ? "rounds and rest" : "all");
  }
}
"""


def build(folder):
    """The program that tells what runs, compiled in `folder`: cases -> ["edge launches"]."""
    from paper_2606_00539_amd import _build as B

    (folder / "tiles.hip").write_text(PROGRAM)
    flags = [f for f in B.HIPCC_FLAGS if f not in ("-shared", "-O3")]
    subprocess.run([B.hipcc(), *flags, "-O1", "-I", CSRC, "-I", os.path.join(ROOT, "include"), "-o",
                    str(folder / "tiles"), str(folder / "tiles.hip")], check=True,
                   capture_output=True)

    def run(cases):
        text = "".join("%s %d %d %d %d\n" % c for c in cases)
        out = subprocess.run([str(folder / "tiles")], input=text, check=True, capture_output=True,
                             text=True, timeout=60).stdout.split("\n")[:-1]
        assert len(out) == len(cases)
        return out
    return run


def loads(groups, rows, seed):
    """`rows` rows over `groups` experts as a router leaves them, every fifth idle."""
    rng = np.random.default_rng(seed)
    p = np.exp(0.8 * rng.standard_normal(groups))
    if groups > 1:
        p[::5] = 0
    return [int(c) for c in rng.multinomial(rows, p / p.sum())]


# K and N of a product (a dgrad's out and in), the rows of its experts (None: one without offsets),
# rows of nobody, and what runs by type of operand; K is no multiple of a step's 64 or 128 values
ROWS = {
    "64 tiles, 70 experts": (72, 88, loads(70, 600, 1), 5, ("64 all", "64 all")),
    "64 tiles, one expert": (136, 80, None, 333, ("64 all", "64 all")),
    "128 tiles, 70 experts": (200, 976, loads(70, 300, 2), 9, ("128 all", "128 all")),
    "128 tiles, 150 experts": (136, 416, loads(150, 700, 3), 0, ("128 all", "128 all")),
    "128 tiles, 8 experts": (360, 1704, loads(8, 1200, 4), 70, ("128 all", "128 all")),
    "128 tiles, one expert": (712, 904, None, 3000, ("128 all", "128 all")),
    "256 tiles, 100 experts": (136, 1208, loads(100, 200, 5), 3, ("256 all", "256 all")),
    "256 tiles, 8 experts": (136, 5752, loads(8, 920, 6), 33, ("256 all", "256 all")),
    "256 tiles, one expert": (136, 392, None, 18500, ("256 all", "256 all")),
    "rounds and rest, 70 experts": (4936, 944, loads(70, 6500, 7), 11,
                                    ("256 rounds and rest", "256 rounds and rest")),
    "rounds and rest, 8 experts": (5128, 5000, loads(8, 4200, 8), 259,
                                   ("256 rounds and rest", "256 rounds and rest")),
    "rounds and rest, one expert": (5128, 3816, None, 10115,
                                    ("256 rounds and rest", "256 rounds and rest")),
}
# out, in, the rows of the experts, and what runs
WGRAD = {
    "whole experts": (200, 136, loads(20, 700, 11), "128 whole"),
    "one expert": (1416, 904, [300], "128 whole"),
    "eighths": (1024, 1160, loads(6, 900, 12), "128 eighths"),
    "uneven eighths": (872, 1272, loads(11, 1500, 13), "128 uneven eighths"),
    "64 uneven eighths": (1160, 872, loads(64, 2000, 14), "128 uneven eighths"),
    "256 tiles, one expert": (5000, 4104, [2100], "256 whole"),
    "256 tiles, uneven eighths": (2104, 2248, [5000, 0, 1300, 2040], "256 uneven eighths"),
    "256 tiles, eighths": (2040, 2304, [2500, 2000, 1700], "256 eighths"),
}


def shape(which, name):
    """(op, rows, groups, out, in) of a case, as the program takes it."""
    if which == "wgrad":
        out, inp, counts, _ = WGRAD[name]
        return "wgrad", sum(counts), len(counts), out, inp
    K, N, counts, pad, _ = ROWS[name]
    rows = pad if counts is None else sum(counts) + pad
    return which, rows, 0 if counts is None else len(counts), *(
        (K, N) if which == "dgrad" else (N, K))


# count, m, n, and what A = X X^T, P and P X run in
BATCH = [
    (1, 40, 40, "64 64 64"),
    (53, 195, 197, "128 128 128"),
    (57, 391, 431, "256 256 256"),
    (51, 663, 1995, "256+128 128 256"),
    (49, 643, 1353, "256+64 128 128"),
    (7, 2112, 2250, "256+128 256+128 256+128"),
    (19, 1154, 1155, "256+64 256+64 256"),
    (4, 923, 4275, "64 64 256+64"),
    (3, 1966, 3098, "128 128 256+128"),
]
