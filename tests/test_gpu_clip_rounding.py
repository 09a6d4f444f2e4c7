"""K11's results bit for bit: the float64 product of a value and the factor, rounded once to the
nearest value of the result's type, ties to even.  The factor is known exactly: with the one norm 1 and
eps 0 it is max_norm."""
import math

import numpy as np
import pytest

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu

# digits of the significand, least exponent of a normal value's frexp, largest value
BF16 = (8, -125, (2.0 - 2.0 ** -7) * 2.0 ** 127)
F32 = (24, -125, (2.0 - 2.0 ** -23) * 2.0 ** 127)


def rounded(v, kind):
    """v (float64) to the nearest of a type's values, ties to even; every step but rint is exact."""
    digits, least, most = kind
    _, e = np.frexp(v)
    e = np.maximum(e, least) - digits           # of the last digit's place
    with np.errstate(over="ignore"):
        r = np.ldexp(np.rint(np.ldexp(v, -e)), e)
    return np.where(np.abs(r) > most, np.copysign(np.inf, v), r)


def test_the_reference_rounds_as_numpy_does():
    rng = np.random.default_rng(1)
    v = rng.standard_normal(20000) * np.exp(rng.uniform(-110, 95, 20000))
    with np.errstate(over="ignore"):
        assert (rounded(v, F32) == v.astype(np.float32)).all()
    assert rounded(np.array([1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8, 1 + 2.0 ** -8 + 2.0 ** -40]),
                   BF16).tolist() == [1.0, 1 + 2.0 ** -6, 1 + 2.0 ** -7]


def clipped(v, factor, into):
    torch = require_gpu()
    from paper_2606_00539_amd import torch_ops

    one = torch.ones(1, dtype=torch.float64, device="cuda")
    out = None if into is None else torch.empty(v.shape, dtype=into, device="cuda")
    norm = torch_ops.clip_gradients([v], factor, out=None if out is None else [out], known=[0],
                                    norms=one, eps=0.0)
    assert float(norm) == 1.0
    return v if out is None else out


def same(got, want):
    return (got.double().cpu().numpy() == want).all()


# just above and below the middle of two bf16 values, by less than fp32 has there, and at it
@pytest.mark.parametrize("by", [2.0 ** -40, -2.0 ** -40, 0.0])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("of", ["bf16", "f32"])
def test_next_to_the_middle(by, in_place, of):
    torch = require_gpu()
    for middle in (0.5 + 2.0 ** -9, 0.5 + 3 * 2.0 ** -9):
        # runs of eight, single values, several exponents down to where bf16 has few digits left
        v = torch.tensor([s * 2.0 ** -k for k in range(132) for s in (1, -1)] + [1.0], device="cuda")
        if of == "bf16":
            v = v.bfloat16()
        elif in_place:
            continue
        want = rounded(v.double().cpu().numpy() * (middle + by), BF16)
        assert same(clipped(v, middle + by, None if in_place else torch.bfloat16), want)


@pytest.mark.parametrize("of", ["bf16", "f32"])
@pytest.mark.parametrize("into", ["bf16", "f32"])
@pytest.mark.parametrize("factor", [1 / 3, math.sqrt(0.5), 0.99999, 1e-3])
def test_many_values(of, into, factor):
    torch = require_gpu()
    types = {"bf16": torch.bfloat16, "f32": torch.float32}
    g = torch.Generator(device="cuda").manual_seed(5)
    n = 4_000_003
    # over the whole range of exponents, and around one
    v = torch.randn(n, generator=g, device="cuda") * torch.exp2(
        torch.randint(-149, 127, (n,), generator=g, device="cuda").float())
    v = torch.cat([v, torch.randn(n, generator=g, device="cuda")])
    v = v[v.isfinite()].to(types[of])
    v = v[v.isfinite()].clone()
    want = rounded(v.double().cpu().numpy() * factor, BF16 if into == "bf16" else F32)
    assert same(clipped(v, factor, types[into]), want)


def test_values_at_the_ends():
    torch = require_gpu()
    top, low = 2.0 ** 128 - 2.0 ** 104, 2.0 ** -149
    v = torch.tensor([top, -top, low, -low, 0.0, -0.0, math.inf, -math.inf], device="cuda")
    for factor in (0.999999, 0.997, 0.5, 1e-30):
        want = rounded(v.double().cpu().numpy()[:6] * factor, BF16)
        got = clipped(v, factor, torch.bfloat16)
        assert same(got[:6], want) and got[6:].tolist() == [math.inf, -math.inf]
        assert (torch.signbit(got[:6]) == torch.signbit(v[:6])).all()
    nan = clipped(torch.tensor([math.nan, 1.0], device="cuda"), 0.5, torch.bfloat16)
    assert nan[0].isnan() and float(nan[1]) == 0.5
