"""Which kernels the grouped products run in, and how a gradient's tiles are shared out.  CPU
only: the rules are host code."""
import os
import subprocess

import pytest

import expert_tiles as T


@pytest.fixture(scope="module")
def tiles(tmp_path_factory):
    return T.build(tmp_path_factory.mktemp("tiles"))


def test_the_shapes_run_where_they_are_meant_to(tiles):
    """A shape that has moved to another kernel leaves its own without a test on the device."""
    names = [(w, n) for w in ("linear", "dgrad", "quantized") for n in T.ROWS]
    want = [T.ROWS[n][4][w == "quantized"] for w, n in names]
    names += [("wgrad", n) for n in T.WGRAD]
    want += [v[3] for v in T.WGRAD.values()]
    got = tiles([T.shape(*n) for n in names])
    assert [(n, g) for n, g, w in zip(names, got, want) if g != w] == []
    every = {"64 all", "128 all", "256 all", "256 rounds and rest"}
    for w in ("linear", "dgrad", "quantized"):
        assert {g for (v, _), g in zip(names, got) if v == w} == every


def test_the_batches_run_where_they_are_meant_to(tiles):
    got = tiles([("batch", count, m, n, 0) for count, m, n, _ in T.BATCH])
    assert got == [want for *_, want in T.BATCH]
    every = {"64", "128", "256", "256+64", "256+128"}
    assert all({g.split()[k] for g in got} == every for k in range(3))


PROGRAM = """
#include <stdio.h>
#include <vector>
#include "groups.h"
// every tile of every group belongs to one workgroup of the launch
int main() {
  for (int num : {1, 2, 3, 7, 8, 9, 64, 65})
    for (int per = 1; per < 300; ++per) {
      std::vector<int> seen(num * per, 0);
      for (int w = 0; w < num * gnmr::slots_of(num, per); ++w) {
        int v = -1, e = -1;
        if (!gnmr::share_of(w, num, per, &v, &e)) continue;
        if (v < 0 || v >= per || e < 0 || e >= num) { printf("%d %d: out of range\\n", num, per); return 1; }
        ++seen[e * per + v];
      }
      for (int n : seen)
        if (n != 1) { printf("%d %d: a tile %d times\\n", num, per, n); return 1; }
    }
  puts("ok");
}
"""


def test_every_tile_of_a_gradient_has_one_workgroup(tmp_path):
    from paper_2606_00539_amd import _build as B

    (tmp_path / "share.hip").write_text(PROGRAM)
    flags = [f for f in B.HIPCC_FLAGS if f not in ("-shared", "-O3")]
    subprocess.run([B.hipcc(), *flags, "-O1", "-I", T.CSRC, "-I", os.path.join(T.ROOT, "include"),
                    "-o", str(tmp_path / "share"), str(tmp_path / "share.hip")], check=True,
                   capture_output=True)
    r = subprocess.run([str(tmp_path / "share")], capture_output=True, text=True, timeout=60)
    assert r.stdout == "ok\n" and r.returncode == 0, r.stdout
