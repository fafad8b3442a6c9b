"""Attention of the local stream in float64, from its definition (numpy).

``rope_fwd`` / ``rope_bwd``: RMSNorm of every head and the rotation of its pairs by
position; ``window_fwd`` / ``window_bwd``: causal attention in a sliding window with
sinks; ``paged_append`` / ``paged_attn``: the paged cache of keys and values and the
attention of the newest token over it.  The bounds beside the results (``mag``,
the sums of absolute values) are what the tests derive their tolerances from.
"""
from __future__ import annotations

import numpy as np


def angles(pos, pairs, theta):
    """[rows, sum(pairs)] angles: pair i of axis a turns by pos_a * theta^(-i / pairs[a])."""
    pos = np.asarray(pos, np.float64)
    return np.concatenate([pos[:, a:a + 1] * theta ** (-np.arange(n) / n) for a, n in enumerate(pairs)]
                          + [np.zeros((len(pos), 0))], 1)


def turn(y, ang):
    """Pairs (2j, 2j+1) of y [rows, heads, dh] turned by ang [rows, <= dh/2]."""
    z = y.copy()
    n = ang.shape[1]
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    a, b = y[..., 0:2 * n:2], y[..., 1:2 * n:2]
    z[..., 0:2 * n:2], z[..., 1:2 * n:2] = a * c - b * s, a * s + b * c
    return z


def rope_fwd(x, w, pos, pairs, theta, eps):
    """x [rows, heads, dh], w [dh] or None."""
    y = x if w is None else w * x / np.sqrt(np.mean(x * x, -1, keepdims=True) + eps)
    return turn(y, angles(pos, pairs, theta))


def rope_bwd(x, w, dz, pos, pairs, theta, eps):
    """(dx, dw or None, sum of the absolute terms of dw)."""
    dy = turn(dz, -angles(pos, pairs, theta))
    if w is None:
        return dy, None, None
    r = 1.0 / np.sqrt(np.mean(x * x, -1, keepdims=True) + eps)
    xh, g = x * r, w * dy
    return (r * (g - xh * np.mean(g * xh, -1, keepdims=True)), np.sum(dy * xh, (0, 1)),
            np.sum(np.abs(dy * xh), (0, 1)))


def visible(i, n, window, n_sink):
    """Which of the keys 0..n-1 query i sees."""
    j = np.arange(n)
    return (j <= i) & ((i - j < window) | (j < n_sink) if window else True)


def _probabilities(q, k, seen):
    s = q @ k.T / np.sqrt(q.shape[-1])
    s = np.where(seen, s, -np.inf)
    m = s.max(-1, keepdims=True)
    e = np.where(seen, np.exp(s - np.where(np.isfinite(m), m, 0.0)), 0.0)
    t = e.sum(-1, keepdims=True)
    return e / np.where(t > 0, t, 1.0)


def window_fwd(q, k, v, window, n_sink):
    """q [B, L, H, dh], k, v [B, L, KV, dh] -> (out, sum_j p_j |v_j|)."""
    B, L, H, _ = q.shape
    g = H // k.shape[2]
    seen = np.stack([visible(i, L, window, n_sink) for i in range(L)])
    out, mag = np.empty_like(q), np.empty_like(q)
    for b in range(B):
        for h in range(H):
            p = _probabilities(q[b, :, h], k[b, :, h // g], seen)
            out[b, :, h], mag[b, :, h] = p @ v[b, :, h // g], p @ np.abs(v[b, :, h // g])
    return out, mag


def window_bwd(q, k, v, do, window, n_sink, u=2.0 ** -8):
    """(dq, dk, dv) and, for each, what rounding p, ds and out to a relative u can move it by."""
    B, L, H, dh = q.shape
    g, sc = H // k.shape[2], 1.0 / np.sqrt(dh)
    seen = np.stack([visible(i, L, window, n_sink) for i in range(L)])
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    eq, ek, ev = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for b in range(B):
        for h in range(H):
            n = h // g
            qh, kh, vh, gh = q[b, :, h], k[b, :, n], v[b, :, n], do[b, :, h]
            p = _probabilities(qh, kh, seen)
            o = p @ vh
            ds = p * (gh @ vh.T - np.sum(gh * o, -1, keepdims=True))
            dq[b, :, h] = ds @ kh * sc
            dk[b, :, n] += ds.T @ qh * sc
            dv[b, :, n] += p.T @ gh
            # out is stored rounded, and Di = do . out made from it
            e = u * (np.abs(ds) + p * np.sum(np.abs(gh * o), -1, keepdims=True))
            eq[b, :, h] = e @ np.abs(kh) * sc
            ek[b, :, n] += e.T @ np.abs(qh) * sc
            ev[b, :, n] += u * (p.T @ np.abs(gh))
    return (dq, dk, dv), (eq, ek, ev)


def paged_append(K, V, table, length, start, q, k, v, w_q, w_k, pos, pairs, theta, eps):
    """K, V [pages, KV, page, dh] with the tokens k, v [rows, KV, dh] written, and the queries.
    Token t of sequence b (start[b] <= t < start[b+1]) goes to row length[b] - (start[b+1] - t)."""
    K, V, page = K.copy(), V.copy(), K.shape[2]
    rows = np.concatenate([np.arange(length[b] - (start[b + 1] - start[b]), length[b])
                           for b in range(len(length))])
    seq = np.repeat(np.arange(len(length)), np.diff(start))
    at = rows[:, None] if pos is None else pos
    kz = rope_fwd(k, w_k, at, pairs, theta, eps)
    for t, (b, r) in enumerate(zip(seq, rows)):
        pg = table[b, r // page]
        K[pg, :, r % page], V[pg, :, r % page] = kz[t], v[t]
    return K, V, rope_fwd(q, w_q, at, pairs, theta, eps)


def paged_attn(q, K, V, table, length, window, n_sink):
    """q [B, H, dh] -> (out, sum_j p_j |v_j|); no rows: zeros."""
    out, mag = np.zeros_like(q), np.zeros_like(q)
    page, g = K.shape[2], q.shape[1] // K.shape[1]
    for b, n in enumerate(length):
        j = np.flatnonzero(visible(n - 1, n, window, n_sink)) if n else np.zeros(0, int)
        if len(j) == 0:
            continue
        k, v = (t[table[b, j // page], :, j % page] for t in (K, V))
        for h in range(q.shape[1]):
            p = _probabilities(q[b, h:h + 1], k[:, h // g], np.ones((1, len(j)), bool))
            out[b, h], mag[b, h] = (p @ v[:, h // g])[0], (p @ np.abs(v[:, h // g]))[0]
    return out, mag
