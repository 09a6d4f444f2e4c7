"""The streamed tiles let a tile's stores be under way while they wait for the next tile's operands, by
the number of memory operations behind those: exactly as many stores have to be issued as they are told
(mm_stream.h).  Read in the compiled code; CPU only."""
import os
import re
import subprocess

import pytest

from paper_2606_00539_amd import _build as B

CSRC = os.path.join(B.PKG, "csrc")
# stores of a tile's end by kernel: what k9_gated.hip passes to mm::stream
STORES = {"k9_linear_streamILi0ELb1": 24, "k9_linear_streamILi0ELb0": 8,
          "k9_linear_streamILi1ELb1": 24, "k9_linear_streamILi1ELb0": 8,
          "k9_dgrad_streamILi0E": 32, "k9_dgrad_streamILi1E": 32}


@pytest.fixture(scope="module")
def code(tmp_path_factory):
    out = tmp_path_factory.mktemp("stream") / "k9.s"
    flags = [f for f in B.HIPCC_FLAGS if f not in ("-shared", "-Wall")]
    subprocess.run([B.hipcc(), *flags, "-I", os.path.join(B.ROOT, "include"),
                    "--cuda-device-only", "-S", "-o", str(out), os.path.join(CSRC, "k9_gated.hip")],
                   check=True, capture_output=True)
    text = out.read_text()
    return {m[1]: m[2] for m in re.finditer(r"\n(_Z\S*_stream\S*):\s*; @.*?\n(.*?)\.Lfunc_end", text,
                                            re.S)}


def test_every_kernel_is_looked_at(code):
    assert len(code) == 12
    assert all(sum(k in n for k in STORES) == 1 for n in code)


@pytest.mark.parametrize("kernel", STORES)
def test_stores_are_as_many_as_the_wait_allows_for(code, kernel):
    for name, body in code.items():
        if kernel not in name:
            continue
        stores = re.findall(r"\n\t(buffer_store\S*|global_store\S*|flat_store\S*|scratch_\S*)", body)
        assert stores == ["buffer_store_dwordx4"] * STORES[kernel], name
        # one block of code has them all: no way around one of them
        blocks = re.split(r"\n\.LBB\d+_\d+:|\n\ts_c?branch\S* ", body)
        counts = [b.count("\tbuffer_store_dwordx4") for b in blocks]
        assert sorted(counts)[-1] == STORES[kernel], (name, counts)
        waits = [int(w) for w in re.findall(r"s_waitcnt vmcnt\((\d+)\)\n", body)]
        assert 12 + STORES[kernel] in waits, (name, waits)
