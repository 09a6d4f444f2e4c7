"""What a gated block's entry points refuse, before anything is launched.  CPU only: device
pointers are only numbers here."""
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


# x 100 x 64, w 4 x 256 x 64, pre 100 x 256, h 100 x 128
def _linear(groups=None, **over):
    _, lib = _lib()
    v = dict(groups=groups or _groups(), x=P, x_stride=64, w=2 * P, pre=3 * P, pre_stride=256,
             h=4 * P, h_stride=128, hidden=128, inp=64, act=0, stream=0)
    v.update(over)
    return lib.gnmr_gated_linear(*v.values())


def _activation(groups=None, **over):
    _, lib = _lib()
    v = dict(groups=groups or _groups(), pre=P, pre_stride=256, h=2 * P, h_stride=128, hidden=128,
             act=0, stream=0)
    v.update(over)
    return lib.gnmr_gated_activation(*v.values())


def _dgrad(groups=None, **over):
    _, lib = _lib()
    v = dict(groups=groups or _groups(), dy=P, dy_stride=64, w=2 * P, pre=3 * P, pre_stride=256,
             dpre=4 * P, dpre_stride=256, out=64, hidden=128, act=0, stream=0)
    v.update(over)
    return lib.gnmr_gated_dgrad(*v.values())


@pytest.mark.parametrize("bad", [
    dict(x=0), dict(x=P + 8), dict(w=0), dict(w=2 * P + 4), dict(pre=3 * P + 2), dict(h=0),
    dict(h=4 * P + 8), dict(x_stride=56), dict(x_stride=68), dict(x_stride=1 << 22),
    dict(pre_stride=248), dict(h_stride=120), dict(hidden=0), dict(hidden=-8), dict(hidden=124),
    dict(inp=0), dict(inp=60), dict(hidden=1 << 21), dict(inp=1 << 22), dict(act=2), dict(act=-1),
    dict(h=P), dict(h=2 * P), dict(h=3 * P), dict(pre=P), dict(pre=2 * P), dict(pre=4 * P - 256),
])
def test_linear_refusals(bad):
    _refused(_linear(**bad))


@pytest.mark.parametrize("bad", [
    dict(pre=0), dict(pre=P + 8), dict(h=0), dict(h=2 * P + 2), dict(pre_stride=128),
    dict(h_stride=132), dict(hidden=12), dict(act=5), dict(h=P), dict(h=P + 100 * 512 - 512),
])
def test_activation_refusals(bad):
    _refused(_activation(**bad))


@pytest.mark.parametrize("bad", [
    dict(dy=0), dict(dy=P + 2), dict(w=0), dict(w=2 * P + 8), dict(pre=0), dict(pre=3 * P + 8),
    dict(dpre=0), dict(dpre=4 * P + 8), dict(dy_stride=56), dict(pre_stride=128),
    dict(dpre_stride=264 + 4), dict(out=4), dict(hidden=0), dict(hidden=1 << 21),
    dict(out=1 << 22), dict(act=7), dict(dpre=P), dict(dpre=2 * P), dict(dpre=3 * P),
])
def test_dgrad_refusals(bad):
    _refused(_dgrad(**bad))


@pytest.mark.parametrize("bad", BAD_GROUPS)
@pytest.mark.parametrize("f", [_linear, _activation, _dgrad])
def test_groups_refusals(f, bad):
    _refused(f(groups=_groups(**bad)))


def test_null_groups():
    _, lib = _lib()
    _refused(lib.gnmr_gated_linear(None, P, 64, 2 * P, None, 0, 3 * P, 128, 128, 64, 0, 0), "groups")
    _refused(lib.gnmr_gated_activation(None, P, 256, 2 * P, 128, 128, 0, 0), "groups")
    _refused(lib.gnmr_gated_dgrad(None, P, 64, 2 * P, 3 * P, 256, 4 * P, 256, 64, 128, 0, 0),
             "groups")


def test_too_many_tiles():
    rows = _groups(rows=2 ** 31 - 257)
    far = dict(x=1 << 56, w=1 << 57, pre=1 << 58, h=1 << 59)
    _refused(_linear(groups=rows, hidden=1 << 20, h_stride=1 << 20, pre_stride=1 << 21, **far),
             "too many")


# x, y, dy, dx 100 rows of 60 values, 64 apart
def _norm(**over):
    B, lib = _lib()
    v = dict(x=P, dtype=B.GNMR_BF16, x_stride=64, weight=2 * P, bias=3 * P, wtype=B.GNMR_F32,
             y=4 * P, y_stride=64, mean=5 * P, rstd=6 * P, rows=100, cols=60, eps=1e-5, stream=0)
    v.update(over)
    return lib.gnmr_layer_norm(*v.values())


def _backward(**over):
    B, lib = _lib()
    v = dict(dy=P, dy_stride=64, x=2 * P, dtype=B.GNMR_F32, x_stride=64, mean=3 * P, rstd=4 * P,
             weight=5 * P, wtype=B.GNMR_BF16, dx=6 * P, dx_stride=64, dw=7 * P, db=8 * P, rows=100,
             cols=60, work=9 * P, bytes=1 << 19, stream=0)
    v.update(over)
    return lib.gnmr_layer_norm_backward(*v.values())


@pytest.mark.parametrize("bad", [
    dict(x=0), dict(y=0), dict(x=P + 1), dict(y=4 * P + 1), dict(weight=2 * P + 2),
    dict(bias=3 * P + 2), dict(mean=5 * P + 2), dict(rstd=6 * P + 1), dict(dtype=2), dict(wtype=-1),
    dict(x_stride=59), dict(y_stride=32), dict(x_stride=(1 << 28) + 1), dict(rows=-1),
    dict(rows=1 << 24), dict(cols=0), dict(cols=16385, x_stride=16385, y_stride=16385),
    dict(eps=-1e-5), dict(eps=float("nan")), dict(eps=float("inf")), dict(y=P), dict(y=2 * P),
    dict(y=3 * P - 64), dict(mean=P + 64), dict(rstd=5 * P), dict(rstd=4 * P + 64),
])
def test_layer_norm_refusals(bad):
    _refused(_norm(**bad))


@pytest.mark.parametrize("bad", [
    dict(dy=0), dict(x=0), dict(mean=0), dict(rstd=0), dict(dy=P + 2), dict(x=2 * P + 2),
    dict(dx=6 * P + 2), dict(weight=5 * P + 1), dict(dw=7 * P + 1), dict(db=8 * P + 1),
    dict(dtype=4), dict(wtype=9), dict(dy_stride=59), dict(x_stride=0), dict(dx_stride=59),
    dict(rows=-5), dict(cols=-1), dict(cols=1 << 15), dict(work=0), dict(work=9 * P + 8),
    dict(bytes=100 * 60 * 8 // 32 - 1), dict(dx=P), dict(dx=2 * P), dict(dw=8 * P), dict(db=2 * P),
    dict(dw=9 * P), dict(work=6 * P), dict(work=2 * P), dict(dx=5 * P),
])
def test_layer_norm_backward_refusals(bad):
    _refused(_backward(**bad))


def test_layer_norm_workspace():
    B, lib = _lib()
    for rows, cols in ((1, 1), (7, 63), (1000, 512), (100000, 16384), (3, 4096)):
        need = B.gnmr_layer_norm_backward_workspace(rows, cols)
        assert need % (8 * cols) == 0 and 0 < need <= rows * 8 * cols
    for bad in ((0, 5), (-1, 5), (5, 0), (5, -2), (5, 16385)):
        assert lib.gnmr_layer_norm_backward_workspace(*bad) == 0


def _gradients(*over):
    B, _ = _lib()
    gs = []
    for k, o in enumerate(over):
        v = dict(in_=(2 + k) * P, out=(2 + k) * P, numel=100, in_dtype=B.GNMR_BF16,
                 out_dtype=B.GNMR_BF16, known=0, reserved=0)
        v.update(o)
        gs.append(B.gnmr_gradient(*v.values()))
    return (B.gnmr_gradient * max(1, len(gs)))(*gs), len(gs)


def _clip(*gradients, **over):
    _, lib = _lib()
    arr, n = _gradients(*gradients)
    v = dict(gradients=arr, num=n, norms=None, num_norms=0, max_norm=1.0, eps=1e-6, norm=P,
             work=P + 4096, bytes=1 << 19, stream=0)
    v.update(over)
    return lib.gnmr_clip_gradients(*v.values())


@pytest.mark.parametrize("bad", [
    dict(in_=0), dict(out=0), dict(numel=-1), dict(numel=(1 << 44) + 1), dict(in_dtype=2),
    dict(out_dtype=-1), dict(known=2), dict(in_=2 * P + 1), dict(out=2 * P + 1),
    dict(out=2 * P + 2), dict(out_dtype=0), dict(out=3 * P), dict(out=3 * P - 100),
    dict(in_=3 * P, out=3 * P), dict(out=P), dict(out=P + 4096), dict(out=P + 8 * P),
])
def test_clip_refuses_a_gradient(bad):
    """The first of two: the second lies at 3 P."""
    if bad.get("out") == 9 * P:
        bad = dict(bad, numel=1 << 43, out=2 * P, in_=2 * P)     # both together past 2^44
        _refused(_clip(bad, dict(in_=1 << 60, out=1 << 60, numel=(1 << 43) + 1)), "2^44")
        return
    _refused(_clip(bad, {}))


@pytest.mark.parametrize("bad", [
    dict(gradients=None), dict(num=-1), dict(num=(1 << 20) + 1), dict(num_norms=3),
    dict(num_norms=-1), dict(norms=5 * P, num_norms=1 << 31), dict(max_norm=-1.0),
    dict(max_norm=float("nan")), dict(eps=-1.0), dict(eps=float("inf")), dict(eps=float("nan")),
    dict(norm=0), dict(norm=P + 4), dict(norms=5 * P + 4, num_norms=1), dict(work=0),
    dict(work=P + 4104), dict(bytes=8), dict(norm=2 * P + 8), dict(work=2 * P),
    dict(norms=P, num_norms=1), dict(norm=P + 4096),
])
def test_clip_refusals(bad):
    _refused(_clip({}, {}, **bad))


def test_nothing_to_do_is_no_error():
    """No rows: accepted without a launch (there is no device here)."""
    B, _ = _lib()
    none = dict(groups=_groups(rows=0))
    assert _linear(**none, x=0, pre=0, h=0) == B.GNMR_OK
    assert _activation(**none, pre=0, h=0) == B.GNMR_OK
    assert _dgrad(**none, dy=0, pre=0, dpre=0) == B.GNMR_OK
    assert _norm(rows=0, x=0, y=0, mean=0, rstd=0) == B.GNMR_OK
    assert _backward(rows=0, dy=0, x=0, dx=0, dw=0, db=0, mean=0, rstd=0, work=0) == B.GNMR_OK
    assert _backward(dx=0, dw=0, db=0, work=0) == B.GNMR_OK


def test_struct_layout():
    B, _ = _lib()
    assert ctypes.sizeof(B.gnmr_gradient) == 40


def test_torch_functions_refuse_host_tensors():
    import torch

    from paper_2606_00539_amd import torch_layers, torch_ops as ops

    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    w = torch.zeros(1, 16, 8, dtype=torch.bfloat16)
    s = torch.zeros(4)
    for f in (lambda: ops.gated_linear(x, w), lambda: ops.gated_activation(x),
              lambda: ops.gated_dgrad(x, w, x), lambda: ops.layer_norm(x),
              lambda: ops.layer_norm_backward(x, x, s, s), lambda: ops.clip_gradients([x], 1.0),
              lambda: torch_layers.layer_norm(x),
              lambda: torch_layers.LayerNorm(8, device="cpu", dtype=torch.float16)):
        with pytest.raises(TypeError):
            f()
    for f in (lambda: ops.clip_gradients([], 1.0), lambda: ops.clip_gradients([x], 1.0, out=[]),
              lambda: ops.clip_gradients([x], 1.0, known=[1]),
              lambda: ops.clip_gradients([x], 1.0, known=[0]),
              lambda: torch_layers.LayerNorm(0, device="cpu"),
              lambda: torch_layers.LayerNorm(16385, device="cpu")):
        with pytest.raises(ValueError):
            f()
