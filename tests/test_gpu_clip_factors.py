"""Clipping by factors that 32 bits do not hold with their full precision (below 2^-126), while the results are ordinary numbers."""
import math

import pytest

torch = pytest.importorskip("torch")

from tests.test_gpu_clip import check, clip, tensors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sizes", [[5000, 17], [100003, 33]])            # one workgroup, two launches
@pytest.mark.parametrize("scale,unscale,max_norm", [(1e36, 2.0 ** -16, 1e-2), (1e35, 1.0, 1e-8), (1e30, 1.0, 1e-12), (1e36, 1.0, 1e-20), (1e35, 1e-41, math.inf), (1e30, 1e-44, 1e-20),
                                                    (1e24, 1e-31, math.inf), (3e35, 1.0, 0.0)])
@pytest.mark.parametrize("out", [None, torch.float32, torch.float16])
def test_factors_below_the_normal_range(sizes, scale, unscale, max_norm, out):
    """As everywhere the factor and the product are rounded once each (check's bound)."""
    unscale = float(torch.tensor(unscale))                               # as the call takes it
    max_norm = float(torch.tensor(max_norm))
    grads = tensors(7, sizes, scale=scale)
    before = [g.clone() for g in grads]
    outs = None if out is None else [torch.full_like(g, 7.0, dtype=out) for g in grads]
    norm = clip(grads, outs, max_norm, unscale)
    check(before, grads if outs is None else outs, norm, max_norm, unscale)


@pytest.mark.parametrize("n", [1000, 100003])
def test_halves_by_such_factors(n):
    grads = tensors(8, [n], torch.float16, 1000.0)
    unscale = float(torch.tensor(1e-39))
    outs = [torch.full((n,), 7.0, device="cuda")]
    check(grads, outs, clip(grads, outs, math.inf, unscale), math.inf, unscale)
