"""The compiled marshalling of a gated block's calls hands the C entry points what ctypes and
plain Python conversions hand them.  CPU only."""
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

    def fields(s):
        return tuple(getattr(s, n) for n, _ in s._fields_)

    def note(name):
        def f(*a):
            a = list(a)
            if "gated" in name:
                a[0] = fields(B.gnmr_groups.from_address(a[0]))
            if "clip" in name:
                a[0] = [fields(g) for g in (B.gnmr_gradient * a[1]).from_address(a[0])]
            got.append([0 if x is None else x for x in a])
            return -7
        return ctypes.CFUNCTYPE(ctypes.c_int, *getattr(lib, name).argtypes)(f)

    for n in B._BLOCK_STEP:
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
        c.bind_block(addresses)
        try:
            yield c, got
        finally:
            c.bind_block(B._addresses(lib, B._BLOCK_STEP))


P, Q = T.data_ptr(), 1 << 40


@pytest.mark.parametrize("off,mask", [(T, None), (None, T), (4096, np.int64(64)), (None, None)])
def test_gated(calls, off, mask):
    c, got = calls
    o = 0 if off is None else int(off.data_ptr() if hasattr(off, "data_ptr") else off)
    m = 0 if mask is None else int(mask.data_ptr() if hasattr(mask, "data_ptr") else mask)
    g = (o or None, m or None, 1 << 33, 7, 1)
    assert c.gated_linear(1 << 33, 7, off, mask, 1, T, 128, Q, None, 0, 5, 1 << 34, 24, 40, 1,
                          None) == -7
    assert got.pop() == [g, P, 128, Q, 0, 0, 5, 1 << 34, 24, 40, 1, 0]
    assert c.gated_linear(1 << 33, 7, off, mask, True, T, 128, Q, T, 1 << 35, 5, 8, 24, 40, 0,
                          77) == -7
    assert got.pop() == [g, P, 128, Q, P, 1 << 35, 5, 8, 24, 40, 0, 77]
    assert c.gated_activation(1 << 33, 7, off, mask, 1, T, 8, Q, 1 << 34, 24, 1, 9) == -7
    assert got.pop() == [g, P, 8, Q, 1 << 34, 24, 1, 9]
    assert c.gated_dgrad(1 << 33, 7, off, mask, 1, T, 8, Q, 3, 1 << 36, T, 16, 24, 40, 0, 0) == -7
    assert got.pop() == [g, P, 8, Q, 3, 1 << 36, P, 16, 24, 40, 0, 0]


def test_layer_norm(calls):
    c, got = calls
    eps = float(np.float32(1e-5))
    assert c.layer_norm(T, 1, 1 << 33, None, None, 0, Q, 1 << 34, None, None, 1 << 35, 60, 1e-5,
                        None) == -7
    assert got.pop() == [P, 1, 1 << 33, 0, 0, 0, Q, 1 << 34, 0, 0, 1 << 35, 60, eps, 0]
    assert c.layer_norm(T, 0, 3, Q, 4, 1, 5, 6, T, 7, 8, 9, np.float32(2.5), 11) == -7
    assert got.pop() == [P, 0, 3, Q, 4, 1, 5, 6, P, 7, 8, 9, 2.5, 11]
    assert c.layer_norm_backward(T, 1 << 33, Q, 1, 1 << 34, 3, T, None, 0, None, 0, None, None,
                                 1 << 35, 60, None, 0, None) == -7
    assert got.pop() == [P, 1 << 33, Q, 1, 1 << 34, 3, P, 0, 0, 0, 0, 0, 0, 1 << 35, 60, 0, 0, 0]
    assert c.layer_norm_backward(1, 2, 3, 0, 4, 5, 6, T, 1, Q, 7, 8, T, 9, 10, Q, 1 << 36,
                                 12) == -7
    assert got.pop() == [1, 2, 3, 0, 4, 5, 6, P, 1, Q, 7, 8, P, 9, 10, Q, 1 << 36, 12]


def test_clip(calls):
    c, got = calls
    assert c.clip_gradients([], None, 0, 1, 0, T, Q, 8, None) == -7
    assert got.pop() == [[], 0, 0, 0, 1.0, 0.0, P, Q, 8, 0]
    many = [(T, Q + k, 1 << 40, 0, 1, k % 2 == 1) for k in range(300)]
    assert c.clip_gradients(many, T, 1 << 20, 2.5, 1e-6, 3, None, 0, 5) == -7
    a = got.pop()
    assert a[0] == [(P, Q + k, 1 << 40, 0, 1, k % 2, 0) for k in range(300)]
    assert a[1:] == [300, P, 1 << 20, 2.5, 1e-6, 3, 0, 0, 5]
    for bad in ([(T, T, 5, 0, 0)], [(T, T, 5, 0, 0, 0, 0)], [5], [(T, T, "x", 0, 0, 0)]):
        with pytest.raises((TypeError, ValueError)):
            c.clip_gradients(bad, None, 0, 1.0, 0.0, T, T, 8, None)
    assert not got


@pytest.mark.parametrize("name,n", [("gated_linear", 16), ("gated_activation", 12),
                                    ("gated_dgrad", 16), ("layer_norm", 14),
                                    ("layer_norm_backward", 18), ("clip_gradients", 9)])
def test_wrong_counts_and_kinds_are_refused(calls, name, n):
    c, got = calls
    for bad in ([1] * (n - 1), [1] * (n + 1), [object()] * n):
        with pytest.raises((TypeError, ValueError)):
            getattr(c, name)(*bad)
    assert not got
