"""Several steps of the orthogonalised update at a time, in products of the short side, against the float64 oracle: short sides of up to 128 in one
workgroup a matrix, longer ones of wide matrices in launches of their own.  Tolerances of X as for a step at a time: 8 2^-24 a step, amplified by the
polynomial's slope a at 0 in the steps behind it."""
import numpy as np
import pytest
import torch

from oracle import more_layer_oracle as mo
from tests.gpu_util import rel_l2
from tests.test_gpu_layers import host
from tests.test_gpu_muon import check, step

pytestmark = pytest.mark.gpu
DEFAULT = [float(np.float32(c)) for c in mo.COEFFICIENTS]


def polynomial_error(count, rows, cols, coefficients, steps):
    """The largest error of X over some of the matrices, and its bound."""
    g = torch.randn(count, rows, cols, device="cuda", generator=torch.Generator(device="cuda").manual_seed(steps + rows))
    theta, m = torch.zeros_like(g), torch.zeros_like(g)
    a, b, c = (float(np.float32(v)) for v in coefficients)
    step(theta, g, m, lr=1.0, momentum=0.0, a=a, b=b, c=c, steps=steps)
    size = np.sqrt(max(1.0, rows / cols))
    err = max(rel_l2(-host(theta[k]) / size, mo.orthogonalise(host(g[k]), steps, float(np.float32(1e-7)), (a, b, c))) for k in {0, count - 1})
    bound = 8 * 2.0 ** -24 * sum(max(abs(a), 1.0) ** k for k in range(steps + 1))
    print("muon", count, rows, cols, coefficients, steps, "error", err, "bound", bound, flush=True)
    return err, bound


@pytest.mark.parametrize("count,rows,cols", [(2, 100, 2000), (12, 200, 2000), (1, 2500, 700)])
@pytest.mark.parametrize("coefficients", [(1.0, -3.0, 6.0), (1.0, -1.0, 6.9), (0.5, 1.0, -8.0)])
def test_muon_of_polynomials_that_could_grow(coefficients, count, rows, cols):
    """Accepted ones whose largest value, at singular values that these matrices do not have, is 1000 times what they take and more: scales are
    made for the largest."""
    err, bound = polynomial_error(count, rows, cols, coefficients, 2)
    assert err <= bound
