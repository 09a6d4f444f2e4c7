"""The compiled marshalling of the expert step's calls hands the C entry points what
ctypes and plain Python conversions hand them.  CPU only."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2606_00539_amd import binding as B

T = torch.zeros(16)


def recording(got):
    """Functions in place of the entry points that note their arguments; -7 is what they
    return."""
    lib, fns = B.load_library(), {}

    def note(name):
        types = getattr(lib, name).argtypes

        def f(*a):
            a = list(a)
            if "quantize_rows" not in name:
                k, s = (6, B.gnmr_newton_schulz) if "ortho" in name else (0, B.gnmr_groups)
                v = s.from_address(a[k])
                a[k] = tuple(getattr(v, n) for n, _ in s._fields_)
            got.append([0 if x is None else x for x in a])
            return -7
        return ctypes.CFUNCTYPE(ctypes.c_int, *types)(f)

    for n in B._EXPERT_STEP:
        fns[n] = note(n)
    return fns, {n: ctypes.cast(f, ctypes.c_void_p).value for n, f in fns.items()}


@pytest.fixture(params=["compiled", "ctypes"])
def calls(request):
    got, lib = [], B.load_library()
    fns, addresses = recording(got)
    if request.param == "ctypes":
        c = B._CtypesCalls(lib)
        c.bind(lib, addresses)
        yield c, got
    else:
        c = B._native()
        if isinstance(c, B._CtypesCalls):
            pytest.skip("the module is not built for this Python")
        c.bind_experts(addresses)
        try:
            yield c, got
        finally:
            c.bind_experts(B._addresses(lib, B._EXPERT_STEP))


P, Q = T.data_ptr(), 1 << 40


@pytest.mark.parametrize("off,mask", [(T, None), (None, T), (4096, np.int64(64)), (None, None)])
def test_grouped(calls, off, mask):
    c, got = calls
    o = 0 if off is None else int(off.data_ptr() if hasattr(off, "data_ptr") else off)
    m = 0 if mask is None else int(mask.data_ptr() if hasattr(mask, "data_ptr") else mask)
    g = (o or None, m or None, 1 << 33, 7, 1)
    assert c.grouped_linear(1 << 33, 7, off, mask, 1, T, 128, Q, 5, 1 << 34, 24, 40, None) == -7
    assert got.pop() == [g, P, 128, Q, 5, 1 << 34, 24, 40, 0]
    assert c.grouped_dgrad(1 << 33, 7, off, mask, True, T, 128, Q, 5, 8, 24, 40, 77) == -7
    assert got.pop() == [g, P, 128, Q, 5, 8, 24, 40, 77]
    assert c.grouped_wgrad(1 << 33, 7, off, mask, 1, T, 8, Q, 16, 3, 1, True, T, 24, 40, 9) == -7
    assert got.pop() == [g, P, 8, Q, 16, 3, 1, 1, P, 24, 40, 9]
    assert c.quantized_linear(1 << 33, 7, off, mask, 1, T, 8, None, Q, 3, T, 16, 24, 40, None, 0,
                              0) == -7
    assert got.pop() == [g, P, 8, 0, Q, 3, P, 16, 24, 40, 0, 0, 0]
    assert c.quantized_linear(1 << 33, 7, off, mask, 1, T, 8, T, Q, 3, T, 16, 24, 40, Q, 1 << 35,
                              0) == -7
    assert got.pop() == [g, P, 8, P, Q, 3, P, 16, 24, 40, Q, 1 << 35, 0]


def test_rows_and_updates(calls):
    c, got = calls
    assert c.quantize_rows(T, 1, 1 << 33, Q, 3, 1 << 34, 40, None) == -7
    assert got.pop() == [P, 1, 1 << 33, Q, 3, 1 << 34, 40, 0]
    assert c.orthogonalize(T, 0, Q, 3, 4, 5, 6, 3.5, -4, np.float32(2.25), 1e-7, 0.5, T, 1 << 35,
                           11) == -7
    z = (6, 3.5, -4.0, 2.25, np.float32(1e-7), 0.5)
    assert got.pop() == [P, 0, Q, 3, 4, 5, z, P, 1 << 35, 11]


@pytest.mark.parametrize("name,n", [("grouped_linear", 13), ("grouped_dgrad", 13),
                                    ("grouped_wgrad", 16), ("quantize_rows", 8),
                                    ("quantized_linear", 17), ("orthogonalize", 15)])
def test_wrong_counts_and_kinds_are_refused(calls, name, n):
    c, got = calls
    for bad in ([1] * (n - 1), [1] * (n + 1), [object()] * n):
        with pytest.raises((TypeError, ValueError)):
            getattr(c, name)(*bad)
    assert not got
