"""The oracle of query/key norm with rotation, gated scan and orthogonalised update: closed forms, gradients against differences."""
import numpy as np
import pytest

from oracle import more_layer_oracle as mo


def directional(f, x, d, h=1e-5):
    return (f(x + h * d) - f(x - h * d)) / (2 * h)


def check_gradients(loss, at, grads, rng, tol=1e-7):
    for i, grad in enumerate(grads):
        d = rng.normal(size=at[i].shape)
        f = lambda z: loss(*(z if j == i else at[j] for j in range(len(at))))  # noqa: E731,B023
        assert abs(directional(f, at[i], d) - (grad * d).sum()) <= tol * np.abs(grad * d).sum(), i


@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
def test_qknorm_products_depend_on_the_distance_alone(pairs):
    rng = np.random.default_rng(1)
    x = np.repeat(rng.normal(size=(1, 1, 1, 2, 12)), 9, 1)                        # the same two heads at nine places
    freq = 0.3 ** np.arange(5)
    y = mo.qknorm(x, None, freq, 1e-9, 10, pairs, positions=[100])
    dot = np.einsum("td,sd->ts", y[0, :, 0, 0], y[0, :, 0, 1])
    assert np.allclose(dot[1:, 1:], dot[:-1, :-1])
    assert np.allclose((y ** 2).mean(-1), 1.0)                                    # a rotation keeps the norm
    assert np.allclose(y[..., 10:], mo.qknorm(x, None, freq, 1e-9, 0, pairs)[..., 10:])


def test_qknorm_as_complex_numbers():
    rng = np.random.default_rng(2)
    x, gamma, freq = rng.normal(size=(2, 3, 1, 1, 8)), rng.normal(1, 0.2, 8), np.array([1.0, 0.1])
    pos = rng.integers(-50, 50, (2, 3))
    y = x * gamma / np.sqrt((x ** 2).mean(-1, keepdims=True) + 1e-3)
    z = (y[..., 0:4:2] + 1j * y[..., 1:4:2]) * np.exp(1j * pos[:, :, None, None, None] * freq)
    got = mo.qknorm(x, gamma, freq, 1e-3, 4, "neighbours", pos, True)
    assert np.allclose(got[..., 0:4:2], z.real) and np.allclose(got[..., 1:4:2], z.imag) and np.allclose(got[..., 4:], y[..., 4:])
    z = (y[..., 0:2] + 1j * y[..., 2:4]) * np.exp(1j * pos[:, :, None, None, None] * freq)
    got = mo.qknorm(x, gamma, freq, 1e-3, 4, "halves", pos, True)
    assert np.allclose(got[..., 0:2], z.real) and np.allclose(got[..., 2:4], z.imag)


@pytest.mark.parametrize("lengths", [None, (5, 0), (2, 9)])
def test_qknorm_gradients_are_the_differences(lengths):
    rng = np.random.default_rng(3)
    x, g, gamma, freq = rng.normal(size=(2, 5, 2, 3, 7)), rng.normal(size=(2, 5, 2, 3, 7)), rng.normal(1, 0.3, 7), rng.normal(size=3)
    loss = lambda x, gamma: (mo.qknorm(x, gamma, freq, 1e-2, 6, "halves", [3, 8], False, lengths) * g).sum()  # noqa: E731
    check_gradients(loss, [x, gamma], mo.qknorm_bwd(x, gamma, freq, 1e-2, 6, "halves", g, [3, 8], False, lengths)[:2], rng)


def test_gatedscan_closed_forms():
    x, zero = np.ones((1, 6, 1, 2)), np.zeros((1, 6, 1, 2))
    lam = np.log(np.expm1(np.array([0.25, 1.0])))                                   # softplus(lam) = 0.25, 1
    h, S = mo.gatedscan(x, zero, 100.0 + zero, lam, 2.0)                            # gates half open: log a = -0.25, -1; u = x
    a = np.exp(-np.array([0.25, 1.0]))
    want = np.sqrt(1 - a ** 2) * (1 - a ** np.arange(1, 7)[:, None]) / (1 - a)      # a geometric sum
    assert np.allclose(h[0, :, 0], want) and np.allclose(S[0, 0], want[-1])
    h, S = mo.gatedscan(x, zero - 1000.0, zero, lam, 2.0, state=np.full((1, 1, 2), 3.0))   # closed: nothing is lost, nothing enters
    assert np.allclose(h, 3.0) and np.allclose(S, 3.0)
    h, S = mo.gatedscan(x, zero, zero, lam, 2.0, lengths=[0], state=np.full((1, 1, 2), 3.0))
    assert not h.any() and np.array_equal(S, np.full((1, 1, 2), 3.0))


@pytest.mark.parametrize("lengths", [None, (7, 0), (3, 9)])
def test_gatedscan_gradients_are_the_differences(lengths):
    rng = np.random.default_rng(4)
    x, r, i, g = (rng.normal(size=(2, 7, 2, 3)) for _ in range(4))
    lam, S0, gS = rng.normal(size=3), rng.normal(size=(2, 2, 3)), rng.normal(size=(2, 2, 3))

    def loss(x, r, i, lam, S0):
        h, S = mo.gatedscan(x, r, i, lam, 1.5, lengths, S0)
        return (h * g).sum() + (S * gS).sum()

    check_gradients(loss, [x, r, i, lam, S0], mo.gatedscan_bwd(x, r, i, lam, 1.5, g, lengths, S0, gS)[:5], rng)


def test_orthogonalise_is_the_polynomial_of_the_singular_values():
    rng = np.random.default_rng(5)
    a, b, c = mo.COEFFICIENTS
    for shape in ((5, 9), (9, 5), (4, 4), (1, 6), (6, 1)):
        u = rng.normal(size=shape)
        U, s, Vt = np.linalg.svd(u, full_matrices=False)
        s = s / np.sqrt((s ** 2).sum())
        for _ in range(5):
            s = a * s + b * s ** 3 + c * s ** 5
        assert np.allclose(mo.orthogonalise(u, 5, 0.0), (U * s) @ Vt)


def test_five_steps_carry_singular_values_near_one():
    """What the binding says of its coefficients."""
    a, b, c = mo.COEFFICIENTS
    s = np.linspace(0.004, 1.0, 200001)
    for _ in range(5):
        s = a * s + b * s ** 3 + c * s ** 5
    print(s.min(), s.max())
    assert s.min() > 0.66 and s.max() < 1.21


def test_muon_of_a_zero_gradient_and_of_a_tall_matrix():
    theta, zero = np.ones((4, 2)), np.zeros((4, 2))
    t, m = mo.muon(theta, zero, zero, 0.1, weight_decay=0.5)
    assert np.allclose(t, 0.95) and not m.any()
    g = np.array([[2.0, 0], [0, 2.0], [0, 0], [0, 0]])
    t, m = mo.muon(zero, g, zero, 1.0, momentum=0.0, steps=1, eps=0.0, coefficients=(1.0, 0.0, 0.0))
    assert np.allclose(t, -np.sqrt(2.0) * g / np.sqrt(8.0)) and np.allclose(m, g)
