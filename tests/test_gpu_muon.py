"""The orthogonalised update through the C ABI against the float64 oracle.

Tolerances, relative to the norm of X.  Operands are two float16 parts, 22 bits and half a step of the last: 2^-23 of each, and the product of the
second parts that is left out is 2^-22 at most: 8 of 2^-24 in all for what a step's products add up (their float32 sums, of at most a few thousand terms
of random signs, are far below that).  The steps behind it amplify small singular values by 3.4445 each:
8 2^-24 (1 + 3.4 + 11.9 + 40.9 + 140.8 + 485) = 3.3e-4 at the very worst after five steps, where all of X is small singular values that
were lost at the first; 8 2^-24 (1 + 3.4) = 2.1e-6 after one.  One part alone would be off by 2^-12 (3.4445)^k, 0.1 and 8e-4.  m is
formed in one fused multiply-add: 2^-24."""
import numpy as np
import pytest
import torch

from oracle import more_layer_oracle as mo
from paper_2207_08393_amd import binding as gb
from tests.gpu_util import rel_l2
from tests.test_gpu_layers import host

pytestmark = pytest.mark.gpu


def bound(steps):
    return 8 * 2.0 ** -24 * sum(3.4445 ** k for k in range(steps + 1))


def step(theta, grad, m, fill=255, **hyper):
    count, rows, cols = (1, *theta.shape) if theta.dim() == 2 else theta.shape
    ws = torch.full((gb.gleam_muon_workspace_bytes(count, rows, cols),), fill, dtype=torch.uint8, device="cuda")
    gb.gleam_muon_step(gb.make_muon(**hyper), theta, grad, m, ws)


def check(count, rows, cols, steps=5, nesterov=True, weight_decay=0.0, momentum=0.95, lr=0.5, gap=0, seed=0, low=None):
    """theta starts small against lr X, so that X's error is what is seen."""
    rng = np.random.default_rng(seed + rows + cols)
    g = rng.normal(size=(count, rows, cols))
    if low:
        g = rng.normal(size=(count, rows, low)) @ rng.normal(size=(count, low, cols)) + 1e-3 * g   # few strong directions
    size = rows * cols + gap
    flat = [torch.full((count * size,), 7.0, device="cuda") for _ in range(3)]
    view = [f.as_strided((count, rows, cols), (size, cols, 1)) for f in flat]
    for t, v in zip(view, (1e-3 * rng.normal(size=g.shape), 1e-2 * g, 1e-2 * rng.normal(size=g.shape))):
        t.copy_(torch.from_numpy(v.astype(np.float32)))
    theta, grad, m = (host(t) for t in view)
    step(*view, lr=lr, steps=steps, nesterov=nesterov, weight_decay=weight_decay, momentum=momentum)
    hyper = dict(lr=lr, momentum=float(np.float32(momentum)), weight_decay=float(np.float32(weight_decay)), nesterov=nesterov, steps=steps, eps=float(np.float32(1e-7)),
                 coefficients=[float(np.float32(c)) for c in mo.COEFFICIENTS])
    for k in range(count):
        t, mm = mo.muon(theta[k], grad[k], m[k], **hyper)
        assert np.abs(host(view[2])[k] - mm).max() <= 2.0 ** -23 * np.abs(mm).max()
        x = mo.muon(theta[k], grad[k], m[k], **{**hyper, "lr": 0.0})[0] - t                    # lr X, without the decay where that is 0
        err = np.linalg.norm(host(view[0])[k] - t) / np.linalg.norm(x)
        print("muon", count, rows, cols, steps, "error", err, "bound", bound(steps), flush=True)
        assert err <= bound(steps), k
    for f, v in zip(flat, view):
        v.fill_(7.0)
        assert bool((f == 7.0).all())                                                    # nothing between the matrices was written
    return err


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 5), (7, 1), (2, 3), (16, 16), (31, 33), (32, 32), (33, 31), (64, 64), (65, 200), (192, 64), (64, 192), (100, 100), (100, 900), (129, 127),
                                       (257, 96), (300, 1000), (1000, 300)])
def test_muon_sizes(rows, cols):
    check(1, rows, cols)
    check(1, rows, cols, steps=1, nesterov=False, weight_decay=0.1)


@pytest.mark.parametrize("count,rows,cols,gap", [(3, 40, 70, 0), (3, 70, 40, 13), (24, 100, 900, 2), (65, 8, 8, 1), (2, 513, 130, 0)])
def test_muon_batches(count, rows, cols, gap):
    check(count, rows, cols, gap=gap)


@pytest.mark.parametrize("steps", [1, 2, 3, 7, 10])
def test_muon_steps(steps):
    check(1, 96, 160, steps=steps, momentum=0.0)


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 7, 10])
@pytest.mark.parametrize("rows,cols", [(100, 2000), (2000, 100)])
def test_muon_of_wide_matrices(rows, cols, steps):
    """Wide enough for several steps at a time."""
    check(12, rows, cols, steps=steps)


@pytest.mark.parametrize("coefficients,steps", [((6.0, -10.0, 5.0), 2), ((1.5, -0.5, 0.0), 8), ((1.0, 0.0, 0.0), 3)])
def test_muon_of_wide_matrices_and_other_polynomials(coefficients, steps):
    g = torch.randn(12, 100, 2000, device="cuda", generator=torch.Generator(device="cuda").manual_seed(steps))
    theta, m = torch.zeros_like(g), torch.zeros_like(g)
    a, b, c = coefficients
    step(theta, g, m, lr=1.0, momentum=0.0, a=a, b=b, c=c, steps=steps)
    for k in (0, 11):
        err = rel_l2(-host(theta[k]), mo.orthogonalise(host(g[k]), steps, float(np.float32(1e-7)), coefficients))
        print("muon", coefficients, steps, "error", err, flush=True)
        assert err <= 8 * 2.0 ** -24 * sum(a ** k for k in range(steps + 1))


def test_muon_of_wide_matrices_with_few_strong_directions():
    check(12, 100, 2000, low=3)


def test_muon_of_few_strong_directions():
    check(1, 200, 300, low=5)
    check(1, 300, 200, low=1)


def test_muon_is_as_good_as_float32_products():
    """Against the same steps in float32 products on the host: not more than twice as far from 64 bits."""
    rng = np.random.default_rng(3)
    g = rng.normal(size=(256, 384)).astype(np.float32)
    theta, grad, m = torch.zeros(256, 384, device="cuda"), torch.from_numpy(g).cuda(), torch.zeros(256, 384, device="cuda")
    step(theta, grad, m, lr=1.0, momentum=0.0)
    want = mo.orthogonalise(g, 5, 1e-7, [float(np.float32(c)) for c in mo.COEFFICIENTS])
    x = g / np.float32(np.sqrt((g.astype(np.float64) ** 2).sum()) + 1e-7)
    a, b, c = (np.float32(v) for v in mo.COEFFICIENTS)
    for _ in range(5):
        A = x @ x.T
        x = a * x + (b * A + c * (A @ A)) @ x
    ours, plain = rel_l2(-host(theta), want), rel_l2(x, want)
    print("muon error", ours, "float32 products", plain)
    assert ours <= 2 * plain


def test_muon_large():
    """More tiles than the chip runs at once, sides that no tile divides; one wide and one tall, at the tolerance of the others."""
    for rows, cols in ((700, 2500), (2500, 700)):
        gen = torch.Generator(device="cuda").manual_seed(rows)
        g = torch.randn(rows, cols, device="cuda", generator=gen)
        theta, m = torch.zeros_like(g), torch.zeros_like(g)
        step(theta, g, m, lr=1.0, momentum=0.0)
        want = mo.orthogonalise(host(g), 5, 1e-7, [float(np.float32(c)) for c in mo.COEFFICIENTS]) * np.sqrt(max(1.0, rows / cols))
        err = rel_l2(-host(theta), want)
        print("muon", rows, cols, "error", err, flush=True)
        assert err <= bound(5)


def test_muon_zero_infinite_and_extreme_gradients():
    g = torch.randn(6, 40, 50, device="cuda")
    g[1], g[2, 3, 4], g[3, 5, 6] = 0.0, float("inf"), float("nan")
    g[4] *= 1e30
    g[5] *= 1e-30
    theta, m = torch.ones_like(g), torch.zeros_like(g)
    step(theta, g, m, lr=1.0, momentum=0.0)
    t = host(theta)
    assert np.array_equal(t[1], np.ones((40, 50))) and np.all(np.isnan(t[2:4]))
    hg = host(g)
    c = [float(np.float32(v)) for v in mo.COEFFICIENTS]
    for k in (0, 4, 5):                                                               # 1e-30 is small against eps and passes nearly as it is
        x = mo.orthogonalise(hg[k], 5, float(np.float32(1e-7)), c)
        assert np.linalg.norm(1.0 - t[k] - x) <= bound(5) * max(np.linalg.norm(x), 1e-3)


@pytest.mark.parametrize("rows,cols", [(40, 50), (100, 300), (40, 1100)])
def test_muon_of_a_cubic(rows, cols):
    """c = 0: no A A.  A step amplifies by 1.5 and not by 3.4, so that the tolerance holds."""
    g = torch.randn(rows, cols, device="cuda", generator=torch.Generator(device="cuda").manual_seed(cols))
    theta, m = torch.zeros_like(g), torch.zeros_like(g)
    step(theta, g, m, lr=1.0, momentum=0.0, a=1.5, b=-0.5, c=0.0, steps=8)
    want = mo.orthogonalise(host(g), 8, float(np.float32(1e-7)), (1.5, -0.5, 0.0))
    assert rel_l2(-host(theta), want) <= bound(8)


@pytest.mark.parametrize("count,rows,cols", [(700, 9, 40), (300, 70, 40), (520, 33, 530)])
def test_muon_of_many_matrices(count, rows, cols):
    """More matrices than the chip has workgroups at once: each gets what it gets alone."""
    gen = torch.Generator(device="cuda").manual_seed(count)
    start = [torch.randn(count, rows, cols, device="cuda", generator=gen) for _ in range(3)]
    all_at_once = [t.clone() for t in start]
    step(*all_at_once, lr=0.1)
    for k in (0, 1, 255, 256, count - 1):
        alone = [t[k].clone() for t in start]
        t, m = mo.muon(*(host(x) for x in alone), lr=0.1, momentum=float(np.float32(0.95)), weight_decay=0.0, nesterov=True, steps=5, eps=float(np.float32(1e-7)),
                       coefficients=[float(np.float32(c)) for c in mo.COEFFICIENTS])
        x = t - host(alone[0])
        assert np.linalg.norm(host(all_at_once[0][k]) - t) <= bound(5) * np.linalg.norm(x) + 2.0 ** -24 * np.linalg.norm(t), k   # theta is rounded
        assert np.abs(host(all_at_once[2][k]) - m).max() <= 2.0 ** -23 * np.abs(m).max()


@pytest.mark.parametrize("count,rows,cols", [(1, 40, 50), (1, 1, 8), (3, 1, 8), (1, 100, 300)])
def test_muon_of_strides_along_sides_of_one(count, rows, cols):
    """Where there is one matrix, or one row, the distance to the next says nothing, and may differ from array to array."""
    gen = torch.Generator(device="cuda").manual_seed(cols)
    start = [torch.randn(count, rows, cols, device="cuda", generator=gen) for _ in range(3)]
    want = [t.clone() for t in start]
    step(*want, lr=0.1)
    for k in range(3):
        mine = [t.clone() for t in start]
        mine[k] = mine[k].as_strided((count, rows, cols), (rows * cols + (5 if count == 1 else 0), cols + (7 if rows == 1 else 0), 1))
        step(*mine, lr=0.1)
        assert all(torch.equal(a, b) for a, b in zip(mine, want))


@pytest.mark.parametrize("rows,cols", [(40, 50), (100, 300)])
def test_muon_with_an_eps_that_is_no_guard(rows, cols):
    """1 / (|u| + eps) passes the range of a float32 where u is zero or tiny; X = u / (|u| + eps) does not."""
    g = torch.randn(2, rows, cols, device="cuda", generator=torch.Generator(device="cuda").manual_seed(rows))
    g[0] = 0.0
    g[1] *= 1e-37
    theta, m = torch.ones_like(g), torch.zeros_like(g)
    step(theta, g, m, lr=1.0, momentum=0.0, eps=2e-38)
    t = host(theta)
    assert np.array_equal(t[0], np.ones((rows, cols)))
    x = mo.orthogonalise(host(g)[1], 5, float(np.float32(2e-38)), [float(np.float32(v)) for v in mo.COEFFICIENTS])
    assert np.linalg.norm(1.0 - t[1] - x) <= bound(5) * np.linalg.norm(x) + 2.0 ** -24 * np.sqrt(rows * cols)   # theta = 1 - X is rounded to 2^-24


def test_muon_repeats_streams_and_graphs():
    """Two steps in a row go on from the state; the same bits on another stream and from a graph."""
    rng = np.random.default_rng(4)
    start = [torch.from_numpy(rng.normal(size=(3, 100, 260)).astype(np.float32)).cuda() for _ in range(3)]
    hyper = dict(lr=0.1, weight_decay=0.1)
    a = [t.clone() for t in start]
    for _ in range(2):
        step(*a, **hyper)
    ht, hg, hm = (host(t) for t in start)
    for k in range(3):
        t, m = ht[k], hm[k]
        for _ in range(2):
            t, m = mo.muon(t, hg[k], m, **hyper)
        assert rel_l2(host(a[0])[k], t) <= bound(5) and rel_l2(host(a[2])[k], m) <= 2.0 ** -22
    side = torch.cuda.Stream()
    b = [t.clone() for t in start]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(2):
            step(*b, fill=0, **hyper)
    side.synchronize()
    assert torch.equal(a[0], b[0]) and torch.equal(a[2], b[2])
    plan, ws = gb.make_muon(**hyper), torch.empty(gb.gleam_muon_workspace_bytes(3, 100, 260), dtype=torch.uint8, device="cuda")
    c = [t.clone() for t in start]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gb.gleam_muon_step(plan, *c, ws)
    for x, y in zip(c, start):
        x.copy_(y)
    d = [t.clone() for t in start]
    for k in range(4):
        c[1].copy_(torch.randn_like(c[1]))
        d[1].copy_(c[1])
        graph.replay()
        torch.cuda.synchronize()
        gb.gleam_muon_step(plan, *d, ws)
        torch.cuda.synchronize()
        assert torch.equal(c[0], d[0]) and torch.equal(c[2], d[2])
