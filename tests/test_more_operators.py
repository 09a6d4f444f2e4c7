"""The performance cases' plain form of clipping, on the CPU: in place with gradients of both types."""
import importlib.util
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def cases(monkeypatch):
    spec = importlib.util.spec_from_file_location(
        "more_operators", os.path.join(ROOT, "perf", "more_operators.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    monkeypatch.setattr(m, "DEV", "cpu")
    return m


def case(dtype, out, **kw):
    return {"kind": "clip", "layers": 2, "d": 12, "ffn": 20, "experts": 0, "dtype": dtype,
            "out": out, "packed": False, "known": 0.0, "ratio": 0.5, **kw}


@pytest.mark.parametrize("out", ["", "bf16", "f32"])
@pytest.mark.parametrize("dtype", ["bf16", "f32", "mixed"])
@pytest.mark.parametrize("packed", [False, True])
def test_destinations_of_one_type_to_a_copy(cases, monkeypatch, dtype, out, packed):
    """A fused copy on the device takes all of its destinations for one type."""
    c = case(dtype, out, packed=packed)
    s = cases.prepare(c, 3)
    was = [g.clone() for g in s["grads"]]
    copied, copy = [], torch._foreach_copy_

    def noted(to, of):
        assert len({t.dtype for t in to}) == 1 and len({t.dtype for t in of}) == 1
        copied.extend(t.data_ptr() for t in to)
        copy(to, of)
    monkeypatch.setattr(torch, "_foreach_copy_", noted)
    got = cases.run(s)
    outs = s["outs"] or s["grads"]
    assert sorted(copied) == sorted(t.data_ptr() for t in outs)
    norm = sum(g.double().square().sum() for g in was).sqrt()
    # a sum of some thousand squares in float64; a product in fp32, rounded once more for bf16
    assert abs(float(got["norm"]) - float(norm)) <= 1e-12 * float(norm)
    factor = min(1.0, s["max_norm"] / (float(norm) + cases.CLIP_EPS))
    assert factor < 1.0
    for o, g in zip(outs, was):
        want = g.double() * factor
        slack = (2.0 ** -23 + (2.0 ** -8 if o.dtype == torch.bfloat16 else 0.0)) * want.abs()
        assert ((o.double() - want).abs() <= slack).all()
