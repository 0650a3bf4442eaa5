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


def gradient(kind, rows, cols):
    rng = np.random.default_rng(rows)
    noise, short = rng.normal(size=(rows, cols)), min(rows, cols)
    if kind == "noise":
        return noise
    if kind == "direction":                                    # a single one, as strong as all of the noise or three times that
        return (3.0 if rows < cols else 1.0) * np.outer(rng.normal(size=rows), rng.normal(size=cols)) + noise
    if kind == "directions":                                   # an eighth of the short side, from 1 to 0.01, over a floor of noise
        few = max(1, short // 8)
        return (rng.normal(size=(rows, few)) * np.logspace(0, -2, few)) @ rng.normal(size=(few, cols)) + 0.3 * noise
    u, _, v = np.linalg.svd(noise, full_matrices=False)        # singular values spread evenly in their logarithm
    return (u * np.logspace(0, -4, short)) @ v


def against_float32(count, g, steps):
    rows, cols = g.shape
    grad = torch.from_numpy(g).cuda().expand(count, rows, cols).contiguous()
    theta, m = torch.zeros_like(grad), torch.zeros_like(grad)
    step(theta, grad, m, lr=1.0, momentum=0.0, steps=steps)
    want = mo.orthogonalise(g, steps, float(np.float32(1e-7)), DEFAULT)
    x = (g / (np.linalg.norm(g.astype(np.float64)) + 1e-7)).astype(np.float32)
    x = np.ascontiguousarray(x.T) if rows > cols else x
    a, b, c = (np.float32(v) for v in mo.COEFFICIENTS)
    for _ in range(steps):
        A = x @ x.T
        x = a * x + (b * A + c * (A @ A)) @ x
    ours, plain = rel_l2(-host(theta[-1]) / np.sqrt(max(1.0, rows / cols)), want), rel_l2(x.T if rows > cols else x, want)
    print("muon", count, rows, cols, steps, "error", ours, "float32 products", plain, "ratio", ours / plain, flush=True)
    assert ours <= 4 * plain


@pytest.mark.parametrize("kind", ["noise", "direction", "directions", "spread"])
@pytest.mark.parametrize("count,rows,cols", [(4, 64, 64), (1, 192, 64), (2, 33, 250), (3, 30, 800), (3, 64, 576), (3, 96, 200), (3, 100, 900), (3, 900, 100), (2, 128, 2000),
                                             (70, 160, 320), (70, 320, 160), (12, 200, 2000), (1, 300, 2500), (1, 512, 2048), (1, 300, 400), (1, 130, 1000)])
def test_muon_against_float32_products(count, rows, cols, kind):
    """X after five steps of the default polynomial against the same steps in float32 products on the host: not more than four times as far from 64
    bits.  A product's operands are off by half a step of 22 bits, 2^-23, each, and the product of the second parts that is left out is 2^-22 at
    most: 2^-21, where operands of float32 are off by 2^-24 each, 2^-23."""
    against_float32(count, gradient(kind, rows, cols).astype(np.float32), 5)


@pytest.mark.parametrize("steps", [3, 4, 7, 10])
@pytest.mark.parametrize("count,rows,cols", [(1, 64, 192), (3, 64, 576), (3, 200, 96), (12, 200, 2000), (1, 140, 170)])
def test_muon_against_float32_products_of_other_step_counts(count, rows, cols, steps):
    for kind in ("noise", "direction", "directions", "spread"):
        against_float32(count, gradient(kind, rows, cols).astype(np.float32), steps)


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 7, 10])
@pytest.mark.parametrize("count,rows,cols,gap", [(12, 200, 2000, 0), (12, 2000, 200, 3), (2, 520, 2100, 1)])
def test_muon_of_wide_matrices_in_launches(count, rows, cols, gap, steps):
    """Short sides of more than 128 and wide enough for several steps at a time; of 7 blocks (short sums of the short side) and of 17."""
    check(count, rows, cols, steps=steps, gap=gap)


@pytest.mark.parametrize("coefficients,steps", [((6.0, -10.0, 5.0), 2), ((6.0, -10.0, 5.0), 1), ((20.0, -20.0, 3.5), 2), ((1.5, -0.5, 0.0), 8), ((1.5, -0.5, 0.0), 5), ((1.0, 0.0, 0.0), 3)])
@pytest.mark.parametrize("count,rows,cols", [(12, 200, 2000), (12, 2000, 200), (3, 90, 400)])
def test_muon_of_wide_matrices_in_launches_and_other_polynomials(count, rows, cols, coefficients, steps):
    """Also a slope that is too large for two steps at a time, and no A A."""
    err, bound = polynomial_error(count, rows, cols, coefficients, steps)
    assert err <= bound


def test_muon_of_wide_matrices_in_launches_with_few_strong_directions():
    check(12, 200, 2000, low=3)
    check(12, 2000, 200, low=1)


def test_muon_of_wide_matrices_in_launches_with_a_matrix_that_is_not_finite():
    """Matrices of one call do not reach each other; a zero one stays."""
    g = torch.randn(12, 200, 2000, device="cuda", generator=torch.Generator(device="cuda").manual_seed(6))
    g[3], g[7, 5, 6] = 0.0, float("nan")
    theta, m = torch.ones_like(g), torch.zeros_like(g)
    step(theta, g, m, lr=1.0, momentum=0.0)
    t = host(theta)
    assert np.array_equal(t[3], np.ones((200, 2000))) and np.all(np.isnan(t[7])) and np.all(np.isfinite(np.delete(t, 7, 0)))
    x = mo.orthogonalise(host(g[8]), 5, float(np.float32(1e-7)), DEFAULT)
    assert np.linalg.norm(1.0 - t[8] - x) <= 8 * 2.0 ** -24 * sum(3.4445 ** k for k in range(6)) * np.linalg.norm(x) + 2.0 ** -24 * np.sqrt(t[8].size)   # 1 - X is rounded
