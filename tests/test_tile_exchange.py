"""The tiles' results change lanes through LDS on their way out.  The compiler must not move a
lane's reads before the other lanes' writes, nor the next pass's writes before the reads: each way
out has a fence of its wavefront between them.  Read in the compiled code; CPU only."""
import os
import re
import subprocess

import pytest

from paper_2606_00539_amd import _build as B

CSRC = os.path.join(B.PKG, "csrc")

PROGRAM = """
#include "mm_tile.h"
using namespace gnmr::mm;
typedef Tile<Bf16, false, false, 128, 128, 2, 128, 2> T;

__device__ u32x2 halves(float a, float b, float c, float d) {
  return u32x2{__float_as_uint(a) >> 16 | (__float_as_uint(b) & 0xFFFF0000u),
               __float_as_uint(c) >> 16 | (__float_as_uint(d) & 0xFFFF0000u)};
}
#define KERNEL(name)                                                             \\
  __global__ __launch_bounds__(kThreads) void name(const float* in, u32x4* out) { \\
    typename T::Acc acc[T::kBM][T::kBN];                                         \\
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;                  \\
    for (int i = 0; i < T::kBM; ++i)                                             \\
      for (int j = 0; j < T::kBN; ++j)                                           \\
        for (int k = 0; k < 16; ++k) acc[i][j][k] = in[threadIdx.x + 64 * k + i + j];
KERNEL(rows16)
  T::out16(acc, wave, lane, [](int, int, float a, float b, float c, float d) {
    return halves(a, b, c, d); },
    [&](int r, int c, const u32x4& v) { out[r * 16 + c / 8] = v; });
}
KERNEL(mirrored16)
  T::out16_mirrored(acc, wave, lane, [](int, int, float a, float b, float c, float d) {
    return halves(a, b, c, d); },
    [&](int r, int c, const u32x4& v) { out[r * 16 + c / 8] = v; });
}
KERNEL(rows32)
  T::out32(acc, wave, lane, [](int) { return 0; },
    [&](int e, f32x4 v, int) {
      out[T::row(e, wave, lane) * 32 + T::col(wave, lane) / 4] = __builtin_bit_cast(u32x4, v); });
}
"""


@pytest.fixture(scope="module")
def code(tmp_path_factory):
    d = tmp_path_factory.mktemp("exchange")
    (d / "exchange.hip").write_text(PROGRAM)
    flags = [f for f in B.HIPCC_FLAGS if f not in ("-shared", "-Wall")]
    subprocess.run([B.hipcc(), *flags, "-I", CSRC, "--cuda-device-only", "-emit-llvm", "-S", "-o",
                    str(d / "exchange.ll"), str(d / "exchange.hip")], check=True,
                   capture_output=True)
    text = (d / "exchange.ll").read_text()
    return {m[1]: m[2] for m in re.finditer(
        r"define [^\n]*amdgpu_kernel void @_Z\d+([a-z]+\d+)P[^\n]*\{\n(.*?)\n\}", text, re.S)}


@pytest.mark.parametrize("name", ["rows16", "mirrored16", "rows32"])
def test_a_fence_between_writes_and_reads(code, name):
    kinds = []
    for line in code[name].split("\n"):
        if "fence syncscope(\"wavefront\")" in line:
            kinds.append("fence")
        elif re.search(r"(load|store) .*addrspace\(3\)", line):
            kinds.append("read" if " load " in line else "write")
    assert "read" in kinds and "write" in kinds
    last = None
    for k in kinds:
        assert not (last in ("read", "write") and k in ("read", "write") and k != last), kinds
        last = k
