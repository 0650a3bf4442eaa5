"""Plain float64 forms of norm and rotation of queries and keys, the gated scan and the orthogonalised update, and of their gradients.

Written from the formulas, pair by pair or token by token; nothing is shared with the library."""
from __future__ import annotations

import numpy as np


def _live(lengths, B, T):
    n = np.full(B, T) if lengths is None else np.clip(np.asarray(lengths), 0, T)
    return np.arange(T)[None, :] < n[:, None]


# ------------------------------------------------------------------------------------------- norm and rotation of queries and keys
def _angles(B, T, freq, positions, each):
    """[B][T][rot/2] in float64: products of two numbers of at most 31 and 24 bits, each rounded once."""
    t = np.arange(T, dtype=np.float64)
    where = np.broadcast_to(t, (B, T)) if positions is None else np.asarray(positions, np.float64).reshape(B, -1) + (0.0 if each else t)
    return where[:, :, None] * np.asarray(freq, np.float64)


def _turn(y, angle, rot, pairs, sign):
    """y [B][T][P][heads][d] with its first rot values turned by sign * angle, pair by pair."""
    out = y.copy()
    for j in range(rot // 2):
        a, b = (j, j + rot // 2) if pairs == "halves" else (2 * j, 2 * j + 1)
        c, s = np.cos(angle[:, :, j])[:, :, None, None], sign * np.sin(angle[:, :, j])[:, :, None, None]
        out[..., a], out[..., b] = y[..., a] * c - y[..., b] * s, y[..., b] * c + y[..., a] * s
    return out


def qknorm(x, gamma, freq, eps, rot, pairs, positions=None, each=False, lengths=None):
    """x [B][T][P][heads][d] -> the same."""
    B, T = x.shape[:2]
    live = _live(lengths, B, T)[:, :, None, None, None]
    x = np.where(live, x, 0.0).astype(np.float64)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    y = x * r * (1.0 if gamma is None else np.asarray(gamma, np.float64))
    return np.where(live, _turn(y, _angles(B, T, freq, positions, each), rot, pairs, 1.0), 0.0)


def qknorm_bwd(x, gamma, freq, eps, rot, pairs, g_out, positions=None, each=False, lengths=None):
    """-> g_x, g_gamma, and the sums of the absolute values that g_gamma's sums are of."""
    B, T = x.shape[:2]
    live = _live(lengths, B, T)[:, :, None, None, None]
    x, g = np.where(live, x, 0.0).astype(np.float64), np.where(live, g_out, 0.0).astype(np.float64)
    g = _turn(g, _angles(B, T, freq, positions, each), rot, pairs, -1.0)
    gg = g * (1.0 if gamma is None else np.asarray(gamma, np.float64))
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    gx = r * (gg - x * r ** 2 * (gg * x).mean(-1, keepdims=True))
    return np.where(live, gx, 0.0), (g * x * r).sum((0, 1, 2, 3)), np.abs(g * x * r).sum((0, 1, 2, 3))


# --------------------------------------------------------------------------------------------------------------------- gated scan
def _sigmoid(v):
    t = np.exp(-np.abs(v))
    return np.where(v < 0, t, 1.0) / (1.0 + t)


def _gates(x, r, i, lam, kappa, live):
    """log a, 1 - a^2, u; where a token is not there a is 1 and u 0."""
    x, r, i = (np.where(live, z, 0.0).astype(np.float64) for z in (x, r, i))
    rate = kappa * (np.maximum(lam, 0.0) + np.log1p(np.exp(-np.abs(lam))))
    log_a = np.where(live, -rate * _sigmoid(r), 0.0)
    return x, r, i, log_a, -np.expm1(2.0 * log_a), np.where(live, _sigmoid(i) * x, 0.0)


def gatedscan(x, r, i, lam, kappa, lengths=None, state=None):
    """x, r, i [B][T][P][C], lam [C] -> h, state [B][P][C]."""
    B, T = x.shape[:2]
    live = _live(lengths, B, T)[:, :, None, None]
    lam = np.asarray(lam, np.float64)
    _, _, _, log_a, lost, u = _gates(x, r, i, lam, kappa, live)
    S = np.zeros(x[:, 0].shape) if state is None else np.array(state, np.float64)
    h = np.zeros(x.shape)
    for t in range(T):
        S = np.exp(log_a[:, t]) * S + np.sqrt(lost[:, t]) * u[:, t]
        h[:, t] = S
    return np.where(live, h, 0.0), S


def gatedscan_bwd(x, r, i, lam, kappa, g_h, lengths=None, state=None, g_state_out=None):
    """-> g_x, g_r, g_i, g_lambda, g_state, and the sums of the absolute values that g_lambda's sums are of.  Where 1 - a^2 is 0, nothing
    enters h, and the product of its root's slope with the gate's goes to 0 with it."""
    B, T = x.shape[:2]
    live = _live(lengths, B, T)[:, :, None, None]
    lam = np.asarray(lam, np.float64)
    x, r, i, log_a, lost, u = _gates(x, r, i, lam, kappa, live)
    S = [np.zeros(x[:, 0].shape) if state is None else np.array(state, np.float64)]
    for t in range(T):
        S.append(np.exp(log_a[:, t]) * S[-1] + np.sqrt(lost[:, t]) * u[:, t])
    E = np.zeros_like(S[0]) if g_state_out is None else np.array(g_state_out, np.float64)
    gx, gr, gi, w, size = (np.zeros(x.shape) for _ in range(5))
    s, si = _sigmoid(r), _sigmoid(i)
    for t in reversed(range(T)):
        G = E + np.where(live[:, t], g_h[:, t], 0.0)
        a, m = np.exp(log_a[:, t]), np.sqrt(lost[:, t])
        slope = np.divide(-log_a[:, t] * a * a, m, out=np.zeros_like(m), where=m > 0)     # dm / d log a times log a
        w[:, t] = G * (u[:, t] * slope + a * S[t] * log_a[:, t])                          # (dL / d log a) log a
        size[:, t] = np.abs(G * u[:, t] * slope) + np.abs(G * a * S[t] * log_a[:, t])
        gx[:, t] = G * m * si[:, t]
        gi[:, t] = G * m * x[:, t] * si[:, t] * _sigmoid(-i[:, t])
        gr[:, t] = w[:, t] * _sigmoid(-r[:, t])
        E = a * G
    ratio = _sigmoid(lam) / (np.maximum(lam, 0.0) + np.log1p(np.exp(-np.abs(lam))))
    only = lambda z: np.where(live, z, 0.0)  # noqa: E731
    return only(gx), only(gr), only(gi), ratio * w.sum((0, 1, 2)), E, ratio * size.sum((0, 1, 2))


# ------------------------------------------------------------------------------------------------------------ orthogonalised update
COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def orthogonalise(u, steps, eps, coefficients=COEFFICIENTS):
    """X of one matrix [rows][cols]."""
    u = np.asarray(u, np.float64)
    x = u / (np.sqrt((u * u).sum()) + eps)
    x = x.T if u.shape[0] > u.shape[1] else x
    a, b, c = coefficients
    for _ in range(steps):
        A = x @ x.T
        x = a * x + (b * A + c * A @ A) @ x
    return x.T if u.shape[0] > u.shape[1] else x


def muon(theta, grad, m, lr, momentum=0.95, weight_decay=0.0, nesterov=True, steps=5, eps=1e-7, coefficients=COEFFICIENTS):
    """One step of one matrix -> theta, m."""
    theta, grad, m = (np.asarray(z, np.float64) for z in (theta, grad, m))
    m = momentum * m + grad
    x = orthogonalise(grad + momentum * m if nesterov else m, steps, eps, coefficients)
    rows, cols = theta.shape
    return (1.0 - lr * weight_decay) * theta - lr * np.sqrt(max(1.0, rows / cols)) * x, m
