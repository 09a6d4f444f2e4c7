"""What the expert step's entry points refuse, before anything is launched.  CPU only:
device pointers are only numbers here."""
import ctypes

import pytest

P = 1 << 20            # an aligned address that nothing reads


def _lib():
    from paper_2606_00539_amd import binding as B

    return B, B.load_library()


def _refused(status, *words):
    B, lib = _lib()
    assert status == B.GNMR_E_INVALID
    message = lib.gnmr_last_error().decode()
    for w in words:
        assert w in message, (w, message)


def _groups(**over):
    B, _ = _lib()
    v = dict(offsets=P, d_mask=None, rows=100, num_groups=4, mask_value=1)
    v.update(over)
    return ctypes.byref(B.gnmr_groups(*v.values()))


BAD_GROUPS = [dict(rows=-1), dict(rows=2 ** 31 - 256), dict(num_groups=0),
              dict(num_groups=65537), dict(offsets=None), dict(offsets=P + 2),
              dict(mask_value=2), dict(mask_value=-1)]


def _linear(name="gnmr_grouped_linear", groups=None, **over):
    _, lib = _lib()
    v = dict(groups=groups or _groups(), x=P, x_stride=64, w=2 * P, y=3 * P, y_stride=128,
             out=128, inp=64, stream=0)
    if name == "gnmr_grouped_dgrad":
        v.update(x_stride=128, y_stride=64)
    v.update(over)
    return getattr(lib, name)(*v.values())


@pytest.mark.parametrize("name", ["gnmr_grouped_linear", "gnmr_grouped_dgrad"])
@pytest.mark.parametrize("bad", [
    dict(x=P + 8), dict(x=0), dict(y=0), dict(y=3 * P + 2), dict(w=0), dict(w=2 * P + 8),
    dict(x_stride=56), dict(x_stride=132), dict(x_stride=1 << 22), dict(y_stride=8),
    dict(out=0), dict(inp=-8), dict(out=124), dict(inp=60), dict(out=1 << 22),
    dict(inp=1 << 22), dict(y=P), dict(y=2 * P), dict(w=3 * P),
])
def test_grouped_rows_refusals(name, bad):
    _refused(_linear(name, **bad))


@pytest.mark.parametrize("bad", BAD_GROUPS)
@pytest.mark.parametrize("name", ["gnmr_grouped_linear", "gnmr_grouped_dgrad"])
def test_groups_refusals(name, bad):
    _refused(_linear(name, groups=_groups(**bad)))


def test_null_groups():
    _, lib = _lib()
    _refused(lib.gnmr_grouped_linear(None, P, 64, 2 * P, 3 * P, 128, 128, 64, 0), "groups")


def test_partly_overlapping_output_is_refused():
    """y starts inside x's last row: the extents count, strides included."""
    end = P + (99 * 200 + 64) * 2
    _refused(_linear(x_stride=200, y=(end - 16) // 16 * 16), "overlaps")


def test_too_many_tiles():
    _refused(_linear(groups=_groups(rows=2 ** 31 - 257), out=1 << 21, y_stride=1 << 21, y=1 << 58,
                     w=1 << 60), "too many")


def _wgrad(groups=None, **over):
    B, lib = _lib()
    v = dict(groups=groups or _groups(), dy=P, dy_stride=128, x=2 * P, x_stride=64, dw=3 * P,
             dtype=B.GNMR_F32, accumulate=0, partials=6 * P, out=128, inp=64, stream=0)
    v.update(over)
    return lib.gnmr_grouped_wgrad(*v.values())


@pytest.mark.parametrize("bad", [
    dict(dy=0), dict(x=0), dict(dw=0), dict(partials=0), dict(dw=3 * P + 8),
    dict(partials=6 * P + 2), dict(dtype=2), dict(dtype=-1), dict(accumulate=2),
    dict(dy_stride=120), dict(x_stride=68), dict(out=4), dict(inp=12), dict(dw=P), dict(dw=2 * P),
    dict(partials=3 * P + 16), dict(partials=P), dict(x=2 * P + 2),
])
def test_wgrad_refusals(bad):
    _refused(_wgrad(**bad))


@pytest.mark.parametrize("bad", BAD_GROUPS)
def test_wgrad_groups_refusals(bad):
    _refused(_wgrad(groups=_groups(**bad)))


def test_num_partials():
    B, lib = _lib()
    assert B.gnmr_grouped_wgrad_num_partials(128, 128) == 1
    assert B.gnmr_grouped_wgrad_num_partials(136, 264) == 2 * 3
    assert lib.gnmr_grouped_wgrad_num_partials(0, 8) == 0
    assert lib.gnmr_grouped_wgrad_num_partials(8, -8) == 0


def _quantize(**over):
    B, lib = _lib()
    v = dict(x=P, dtype=B.GNMR_BF16, stride=64, codes=2 * P, scale=3 * P, rows=100, cols=64,
             stream=0)
    v.update(over)
    return lib.gnmr_quantize_rows(*v.values())


@pytest.mark.parametrize("bad", [
    dict(x=0), dict(codes=0), dict(scale=0), dict(x=P + 8), dict(codes=2 * P + 4),
    dict(scale=3 * P + 1), dict(dtype=3), dict(stride=56), dict(stride=68), dict(rows=-1),
    dict(rows=1 << 31), dict(cols=0), dict(cols=12), dict(cols=1 << 17, stride=1 << 17),
    dict(codes=P), dict(scale=2 * P), dict(scale=P + 64),
])
def test_quantize_refusals(bad):
    _refused(_quantize(**bad))


def _quantized(groups=None, **over):
    _, lib = _lib()
    v = dict(groups=groups or _groups(), x=P, x_stride=64, x_scale=None, codes=2 * P,
             w_scale=3 * P, y=4 * P, y_stride=128, out=128, inp=64, work=5 * P, bytes=6800,
             stream=0)
    v.update(over)
    return lib.gnmr_quantized_linear(*v.values())


@pytest.mark.parametrize("bad", [
    dict(x=0), dict(codes=0), dict(w_scale=0), dict(y=0), dict(work=0), dict(bytes=6799),
    dict(work=5 * P + 8), dict(codes=2 * P + 4), dict(w_scale=3 * P + 2), dict(x=P + 8),
    dict(x_scale=7 * P + 2), dict(x_scale=7 * P, x=P + 4), dict(y=P), dict(y=2 * P),
    dict(y=3 * P), dict(work=P), dict(work=2 * P), dict(work=4 * P), dict(out=100), dict(inp=20),
    dict(inp=1 << 17, x_stride=1 << 17), dict(x_stride=60), dict(x_scale=4 * P),
])
def test_quantized_refusals(bad):
    _refused(_quantized(**bad))


def test_quantized_workspace():
    B, lib = _lib()
    assert B.gnmr_quantized_linear_workspace(100, 64) == 6800
    assert B.gnmr_quantized_linear_workspace(3, 72) == 3 * (80 + 4)
    assert lib.gnmr_quantized_linear_workspace(-1, 64) == 0


def _ortho(**over):
    B, lib = _lib()
    z = dict(steps=5, a=3.4445, b=-4.775, c=2.0315, eps=1e-7, scale=1.0)
    z.update({k: over.pop(k) for k in list(over) if k in z})
    v = dict(x=P, dtype=B.GNMR_BF16, out=2 * P, rows=64, cols=96, count=2,
             settings=ctypes.byref(B.gnmr_newton_schulz(*z.values())), work=4 * P,
             bytes=1 << 30, stream=0)
    v.update(over)
    return lib.gnmr_orthogonalize(*v.values())


@pytest.mark.parametrize("bad", [
    dict(x=0), dict(out=0), dict(work=0), dict(settings=None), dict(dtype=5), dict(rows=0),
    dict(cols=-3), dict(rows=65537), dict(count=-1), dict(count=65536), dict(steps=0),
    dict(steps=101), dict(a=float("nan")), dict(b=float("inf")), dict(c=float("-inf")),
    dict(eps=-1.0), dict(eps=float("nan")), dict(scale=float("inf")), dict(bytes=1000),
    dict(work=4 * P + 16), dict(x=P + 1), dict(out=P), dict(out=4 * P), dict(work=P),
    dict(out=2 * P + 1),
])
def test_orthogonalize_refusals(bad):
    _refused(_ortho(**bad))


def test_orthogonalize_workspace():
    B, lib = _lib()
    one = B.gnmr_orthogonalize_workspace(60, 100, 1)
    assert one == B.gnmr_orthogonalize_workspace(100, 60, 1) > 0
    assert B.gnmr_orthogonalize_workspace(60, 100, 7) > 6 * (one - 1024)
    for bad in ((0, 5, 1), (5, 0, 1), (5, 5, 0), (-1, 5, 1)):
        assert lib.gnmr_orthogonalize_workspace(*bad) == 0


def test_nothing_to_do_is_no_error():
    """No rows, no matrices: accepted without a launch (there is no device here)."""
    B, lib = _lib()
    none = _groups(rows=0)
    assert _linear(groups=none, x=0, y=0) == B.GNMR_OK
    assert _linear("gnmr_grouped_dgrad", groups=none, x=0, y=0) == B.GNMR_OK
    assert _quantized(groups=none, x=0, y=0, work=0, bytes=0) == B.GNMR_OK
    assert _quantize(rows=0, x=0, codes=0, scale=0) == B.GNMR_OK
    assert _ortho(count=0) == B.GNMR_OK


def test_struct_layouts():
    B, _ = _lib()
    assert ctypes.sizeof(B.gnmr_groups) == 32
    assert ctypes.sizeof(B.gnmr_newton_schulz) == 24


def test_torch_functions_refuse_host_tensors():
    import torch

    from paper_2606_00539_amd import torch_ops as ops

    x, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(1, 8, 8, dtype=torch.bfloat16)
    q = torch.zeros(8, 8, dtype=torch.int8)
    for f in (lambda: ops.grouped_linear(x, w), lambda: ops.grouped_dgrad(x, w),
              lambda: ops.grouped_wgrad(x, x), lambda: ops.quantize_rows(x),
              lambda: ops.quantized_linear(x, q, torch.zeros(8)),
              lambda: ops.orthogonalize(x)):
        with pytest.raises(TypeError):
            f()
