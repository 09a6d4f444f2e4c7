"""The powers of two that K8 holds its Gram matrix and polynomial with, compiled for the
CPU: nothing that an update can reach passes fp16's largest value while the singular values
stay below 15.9, and the usual coefficients keep 2^12."""
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_00539_amd", "csrc")

PROGRAM = """
#include <cstdio>
#include "k8_range.h"
int main() {
  float a, b, c;
  int steps;
  while (scanf("%f %f %f %d", &a, &b, &c, &steps) == 4) {
    const gnmr::HeldExponents e = gnmr::held_exponents(a, b, c, steps);
    printf("%d %d\\n", e.a, e.p);
  }
}
"""


@pytest.fixture(scope="module")
def exponents(tmp_path_factory):
    d = tmp_path_factory.mktemp("range")
    (d / "range.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined",
                    "-fno-sanitize-recover=undefined", "-I", CSRC, "-o", str(d / "range"),
                    str(d / "range.cpp")], check=True)

    def run(cases):
        text = "".join("%r %r %r %d\n" % c for c in cases)
        out = subprocess.run([str(d / "range")], input=text, check=True, capture_output=True,
                             text=True, timeout=60).stdout.split("\n")[:-1]
        assert len(out) == len(cases)
        return [tuple(map(int, line.split())) for line in out]
    return run


def test_usual_coefficients_keep_their_scale(exponents):
    cases = [(3.4445, -4.775, 2.0315, k) for k in (1, 5, 100)]
    cases += [(1.5, -0.5, 0.0, 30), (1.875, -1.25, 0.375, 30), (0.0, 0.0, 0.0, 5)]
    assert exponents(cases) == [(12, 12)] * len(cases)


def test_nothing_passes_the_largest_half(exponents):
    rng = np.random.default_rng(1)
    cases = [(5.2, -0.2, 0.0, 2), (16.0, 0.0, 0.0, 1), (36.0, 0.0, 0.0, 2), (40.0, 0.0, -25.0, 2),
             (8.28, -23.6, 17.3, 8), (3e38, -3e38, 3e38, 3), (-3e38, 0.0, 0.0, 1)]
    for _ in range(600):
        a, b, c = rng.standard_normal(3) * np.exp(rng.uniform(-2, 4, 3))
        cases.append((float(a), float(b), float(c), int(rng.integers(1, 12))))
    held = 0
    for (a, b, c, steps), (ea, ep) in zip(cases, exponents(cases)):
        assert ea <= 12 and ep <= 12
        sigma = np.linspace(0, 1, 5001)
        for _ in range(steps):
            if np.abs(sigma).max() >= 15.9:
                break
            s = sigma * sigma
            p = a + b * s + c * s * s
            assert s.max() * 2.0 ** ea < 65504 and np.abs(p).max() * 2.0 ** ep < 65504, (a, b, c)
            sigma = sigma * p
            held += 1
    assert held > 1000
