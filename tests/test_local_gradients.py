"""Gradients of the windowed attention against differences of its forward, along the gradient itself, and what that
tells apart: on the float64 oracle with results rounded to bf16 the right gradient passes, and wrong ones do not.

A step h along the gradient d (|d| = 1) moves sum(do . out) by 2 h |d| between its two ends.  Off that by: the
curvature, which grows as h^2 (oracle, h = 1, 2, 4: 0.2, 0.9 and 3 % of it; 1 % is allowed at h = 1), the gradient's
own rounding (below 1 %), and the roundings of out and of its probabilities at both ends, each at most 2^-8 of out and
of random sign: four times their root sum of squares, twice."""
import numpy as np
import pytest
import torch

from oracle import local as OL

CASES = [(1, 90, 1, 1, 30, 2), (2, 300, 4, 2, 150, 5), (1, 257, 2, 1, 0, 0)]  # batch, L, heads, kv, window, sinks


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).bfloat16().double().numpy()


def inputs(case, seed=1):
    B, L, H, KV, _, _ = case
    rng = np.random.default_rng(seed)
    return [bf16(rng.standard_normal((B, L, n, 64)).astype(np.float32)) for n in (H, KV, KV, H)]  # q, k, v, do


def difference(forward, x, i, d, do):
    """What a step along d changes by, by the forward and by d, and how far apart these may be."""
    ends = []
    for s in (1.0, -1.0):
        y = [t.copy() for t in x]
        y[i] = bf16(y[i] + s * d / np.linalg.norm(d))
        ends.append((y[i], forward(*y)))
    (xa, a), (xb, b) = ends
    want = ((xa - xb) * d).sum()
    noise = 2.0 ** -8 * np.sqrt(((a ** 2 + b ** 2) * do ** 2).sum())
    return ((a - b) * do).sum(), want, 0.02 * abs(want) + 2 * 4 * noise


@pytest.mark.parametrize("case", CASES)
def test_wrong_gradients_show(case):
    _, L, H, KV, window, n_sink = case
    q, k, v, do = inputs(case)
    forward = lambda *x: bf16(OL.window_fwd(*x, window, n_sink)[0])
    right = [bf16(d) for d in OL.window_bwd(q, k, v, do, window, n_sink)[0]]
    # without Di: dS = P dP
    no_di = [np.zeros_like(q), np.zeros_like(k)]
    seen = np.stack([OL.visible(i, L, window, n_sink) for i in range(L)])
    for b in range(q.shape[0]):
        for h in range(H):
            g = h // (H // KV)
            ds = OL._probabilities(q[b, :, h], k[b, :, g], seen) * (do[b, :, h] @ v[b, :, g].T) / 8
            no_di[0][b, :, h] = ds @ k[b, :, g]
            no_di[1][b, :, g] += ds.T @ q[b, :, h]
    for i, d in enumerate(right):
        got, want, bar = difference(forward, (q, k, v), i, d, do)
        assert abs(got - want) <= bar, (i, got, want, bar)
        for wrong in [-d, 2 * d, 0.5 * d] + no_di[i:i + 1]:
            got, want, bar = difference(forward, (q, k, v), i, wrong, do)
            assert abs(got - want) > bar, (i, got, want, bar)
