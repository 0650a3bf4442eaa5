"""Plain float64 forms of layer norm, dropout and linear attention with a decay for each head, and of their gradients.

Written from the formulas, element by element or token by token; nothing is shared with the library."""
from __future__ import annotations

import numpy as np


def layer_norm(x, gamma, beta, eps):
    """x [rows][n] -> y, mean, rstd."""
    x = np.asarray(x, np.float64)
    mean = x.mean(1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    y = y * (1.0 if gamma is None else np.asarray(gamma, np.float64)) + (0.0 if beta is None else np.asarray(beta, np.float64))
    return y, mean, rstd


def layer_norm_bwd(x, gamma, mean, rstd, g):
    """Gradients from the statistics of the forward pass -> g_x, g_gamma, g_beta."""
    x, g, mean, rstd = (np.asarray(a, np.float64) for a in (x, g, mean, rstd))
    xh = (x - mean[:, None]) * rstd[:, None]
    gg = g * (1.0 if gamma is None else np.asarray(gamma, np.float64))
    gx = rstd[:, None] * (gg - gg.mean(1, keepdims=True) - xh * (gg * xh).mean(1, keepdims=True))
    return gx, (g * xh).sum(0), g.sum(0)


def philox(counter, key):
    """Philox 4x32-10 (Salmon, Moraes, Dror, Shaw 2011) in Python integers: four words from a counter of four and a key of two."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def dropout_mask(rows, n, p, seed, offset, first_row=0):
    """(kept [rows][n], factor) of rows first_row, first_row + 1, ..."""
    low = 0xFFFFFFFF
    offset &= 0xFFFFFFFFFFFFFFFF
    kept = int(np.floor(65536 * (1 - float(np.float32(p))) + 0.5))
    mask = np.zeros((rows, n), bool)
    blocks = {}
    for r in range(rows):
        for c in range(n):
            e = (first_row + r) * n + c
            if e >> 3 not in blocks:
                w = philox((e >> 3 & low, e >> 35, offset & low, offset >> 32), (seed & low, seed >> 32))
                blocks = {e >> 3: [h for x in w for h in (x & 0xFFFF, x >> 16)]}
            mask[r, c] = blocks[e >> 3][e & 7] < kept
    return mask, 65536.0 / kept if kept else 0.0


def _wide(x, H):
    """Heads of [B][T][P][h][d] repeated to H."""
    return np.repeat(np.asarray(x, np.float64), H // x.shape[3], 3)


def _shared(g, heads):
    """Sum over the output heads that use one head."""
    B, T, P, H, d = g.shape
    return g.reshape(B, T, P, heads, H // heads, d).sum(4)


def _live(lengths, B, T):
    n = np.full(B, T) if lengths is None else np.clip(np.asarray(lengths), 0, T)
    return np.arange(T)[None, :] < n[:, None]


def linattn(q, k, v, log_decay, scale, lengths=None, state=None):
    """q, k [B][T][P][h][dk], v [B][T][P][h][dv], log_decay [H] -> o [B][T][P][H][dv], state [B][P][H][dk][dv]."""
    H = len(log_decay)
    B, T, P = q.shape[:3]
    live = _live(lengths, B, T)
    q, k, v = (np.where(live[:, :, None, None, None], _wide(x, H), 0.0) for x in (q, k, v))
    decay = np.exp(np.asarray(log_decay, np.float64))[:, None, None]
    S = np.zeros((B, P, H, k.shape[4], v.shape[4])) if state is None else np.array(state, np.float64)
    o = np.zeros((B, T, P, H, v.shape[4]))
    for t in range(T):
        S = np.where(live[:, t, None, None, None, None], decay * S + k[:, t, ..., :, None] * v[:, t, ..., None, :], S)
        o[:, t] = scale * (q[:, t, ..., None, :] @ S)[..., 0, :]
    return o, S


def linattn_bwd(q, k, v, log_decay, scale, g_o, lengths=None, state=None, g_state_out=None):
    """-> g_q, g_k, g_v, g_state."""
    H = len(log_decay)
    B, T, P = q.shape[:3]
    heads = q.shape[3], k.shape[3], v.shape[3]
    live = _live(lengths, B, T)
    q, k, v, g = (np.where(live[:, :, None, None, None], _wide(x, H), 0.0) for x in (q, k, v, g_o))
    g = scale * g
    decay = np.exp(np.asarray(log_decay, np.float64))[:, None, None]
    S = np.zeros((B, P, H, k.shape[4], v.shape[4])) if state is None else np.array(state, np.float64)
    G = np.zeros_like(S) if g_state_out is None else np.array(g_state_out, np.float64)
    gq, gk, gv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for t in range(T):
        S = np.where(live[:, t, None, None, None, None], decay * S + k[:, t, ..., :, None] * v[:, t, ..., None, :], S)
        gq[:, t] = (S @ g[:, t, ..., :, None])[..., 0]
    for t in reversed(range(T)):
        on = live[:, t, None, None, None]
        N = G + q[:, t, ..., :, None] * g[:, t, ..., None, :]
        gk[:, t] = np.where(on, (N @ v[:, t, ..., :, None])[..., 0], 0.0)
        gv[:, t] = np.where(on, (k[:, t, ..., None, :] @ N)[..., 0, :], 0.0)
        G = np.where(on[..., None], decay * N, G)
    return _shared(gq, heads[0]), _shared(gk, heads[1]), _shared(gv, heads[2]), G
