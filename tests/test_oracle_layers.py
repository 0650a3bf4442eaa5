"""The oracle of the sequence-layer operators: closed forms, known answers of the generator, gradients against differences."""
import numpy as np
import pytest

from oracle import layer_oracle as lo


def directional(f, x, d, h=1e-5):
    return (f(x + h * d) - f(x - h * d)) / (2 * h)


def test_layer_norm_rows_have_zero_mean_and_unit_variance():
    rng = np.random.default_rng(1)
    x = rng.normal(3.0, 2.0, (5, 37))
    y, mean, rstd = lo.layer_norm(x, None, None, 1e-12)
    assert np.allclose(y.mean(1), 0, atol=1e-12) and np.allclose((y ** 2).mean(1), 1, atol=1e-9)
    assert np.allclose(x, y / rstd[:, None] + mean[:, None])


def test_layer_norm_gradients_are_the_differences():
    rng = np.random.default_rng(2)
    x, g = rng.normal(0.5, 1.3, (4, 11)), rng.normal(size=(4, 11))
    gamma, beta, eps = rng.normal(1, 0.2, 11), rng.normal(size=11), 1e-3
    loss = lambda x, a, b: (lo.layer_norm(x, a, b, eps)[0] * g).sum()  # noqa: E731
    _, mean, rstd = lo.layer_norm(x, gamma, beta, eps)
    gx, gg, gb = lo.layer_norm_bwd(x, gamma, mean, rstd, g)
    for grad, f, at in ((gx, lambda z: loss(z, gamma, beta), x), (gg, lambda z: loss(x, z, beta), gamma), (gb, lambda z: loss(x, gamma, z), beta)):
        d = rng.normal(size=at.shape)
        assert abs(directional(f, at, d) - (grad * d).sum()) <= 1e-7 * np.abs(grad * d).sum()


def test_philox_known_answers():
    """The three vectors that the method's authors give for 4x32-10."""
    F = 0xFFFFFFFF
    assert lo.philox((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert lo.philox((F, F, F, F), (F, F)) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert lo.philox((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0)) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_dropout_keeps_the_stated_share():
    mask, factor = lo.dropout_mask(64, 64, 0.25, 7, 3)
    assert factor == 65536 / 49152
    assert abs(mask.mean() - 0.75) < 5 * np.sqrt(0.25 * 0.75 / 4096)      # five standard deviations of 4096 draws
    assert not np.array_equal(mask, lo.dropout_mask(64, 64, 0.25, 7, 4)[0]) and lo.dropout_mask(3, 5, 1.0, 1, 1)[1] == 0.0
    assert lo.dropout_mask(3, 5, 0.0, 1, 1)[0].all() and not lo.dropout_mask(3, 5, 1.0, 1, 1)[0].any()


def _case(rng, B=2, T=7, P=2, H=4, heads=(4, 2, 1), dk=3, dv=5):
    q, k, v = (rng.normal(size=(B, T, P, h, d)) for h, d in zip(heads, (dk, dk, dv)))
    return q, k, v, -rng.uniform(0.01, 1.0, H), rng.normal(size=(B, P, H, dk, dv)), rng.normal(size=(B, T, P, H, dv))


def test_linattn_is_the_masked_product():
    q, k, v, a, S0, _ = _case(np.random.default_rng(3))
    lengths = np.array([7, 4])
    o, S = lo.linattn(q, k, v, a, 0.7, lengths, S0)
    for b, h in ((0, 1), (1, 3)):
        n = lengths[b]
        Q, K, V = q[b, :n, 1, h], k[b, :n, 1, h // 2], v[b, :n, 1, 0]
        i = np.arange(n)
        W = np.where(i[:, None] >= i, np.exp(a[h] * (i[:, None] - i)), 0.0)
        ref = 0.7 * ((Q @ K.T * W) @ V + np.exp(a[h] * (i + 1))[:, None] * (Q @ S0[b, 1, h]))
        assert np.allclose(o[b, :n, 1, h], ref) and not o[b, n:].any()
        assert np.allclose(S[b, 1, h], np.exp(a[h] * n) * S0[b, 1, h] + (K * np.exp(a[h] * (n - 1 - i))[:, None]).T @ V)


@pytest.mark.parametrize("lengths", [None, (7, 0), (3, 9)])
def test_linattn_gradients_are_the_differences(lengths):
    rng = np.random.default_rng(4)
    q, k, v, a, S0, g = _case(rng)
    gS = rng.normal(size=S0.shape)

    def loss(q, k, v, S0):
        o, S = lo.linattn(q, k, v, a, 0.7, lengths, S0)
        return (o * g).sum() + (S * gS).sum()

    grads = lo.linattn_bwd(q, k, v, a, 0.7, g, lengths, S0, gS)
    at = [q, k, v, S0]
    for i, grad in enumerate(grads):
        d = rng.normal(size=at[i].shape)
        f = lambda z: loss(*(z if j == i else at[j] for j in range(4)))  # noqa: E731,B023
        assert abs(directional(f, at[i], d) - (grad * d).sum()) <= 1e-7 * np.abs(grad * d).sum()
