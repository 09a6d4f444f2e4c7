"""How near K8 comes to the definition in float64, where its roundings could all go one way: in an
update much wider than high the singular values are nearly equal, so the diagonals of A = X X^T
and of P are, and would be rounded alike in every row and step.

Tolerance in the 2-norm.  X, A and P are rounded to fp16 in each of five steps, by 2^-11 of a value
at most and so by 2^-11 / sqrt(3) = 2.8e-4 in the mean square, independently from value to value
once the diagonals are kept whole; a step multiplies a relative error of a singular value by
|1 + 2 s p'(s) / p(s)|, which is below 1.55 for squares s to 1.2 (and rises to 5 at the largest that
occurs, 1.45, where few are at a time): sqrt(15) * 2.8e-4 * 1.55 = 1.7e-3.  The result's rounding to bf16 is 2^-8 at most, 1.66e-3 in the mean square over values
of all sizes.  Together 2.4e-3."""
import numpy as np
import pytest

from gpu_util import require_gpu
from oracle import experts as X

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("strong", [False, True])
@pytest.mark.parametrize("m,n", [(8, 3000), (32, 1673), (32, 13824), (1673, 32), (40, 5000), (35, 265),
                                 (33, 86), (242, 2577), (280, 2108), (1673, 300), (128, 128),
                                 (256, 688), (700, 1300)])
def test_error(m, n, strong, dtype):
    torch = require_gpu()
    from paper_2606_00539_amd import torch_ops

    rng = np.random.default_rng(m * 100003 + n)
    k = min(m, n)
    g = rng.standard_normal((m, n))
    if strong:
        r = max(1, k // 32)
        g += 0.5 * (rng.standard_normal((m, r)) / np.sqrt(np.arange(1, r + 1))) @ \
            rng.standard_normal((r, n))
    g = (1e-4 * g).astype(np.float32)
    if dtype == "bf16":
        g = X.bf16(g)
    want = X.orthogonalize(g, 5, (3.4445, -4.775, 2.0315), 1e-7)
    gt = torch.from_numpy(g).cuda()
    got = torch_ops.orthogonalize(gt.to(torch.bfloat16) if dtype == "bf16" else gt)
    error = np.linalg.norm(got.double().cpu().numpy() - want) / np.linalg.norm(want)
    print("orthogonalize", m, n, strong, dtype, "error %.5f" % error, flush=True)
    assert error <= 2.4e-3
