"""The float64 attention of the local stream against differences, torch and itself."""
import numpy as np
import pytest
import torch

from oracle import local as OL


def _difference(f, x, g, eps=1e-6):
    """d sum(g f(x)) / dx by central differences."""
    d = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        for s in (1, -1):
            y = x.copy()
            y[i] += s * eps
            d[i] += s * np.sum(g * f(y)) / (2 * eps)
    return d


@pytest.mark.parametrize("pairs", [(4,), (2, 2), (1, 2, 1), (3,), ()])
@pytest.mark.parametrize("norm", [False, True])
def test_rope_gradients(pairs, norm):
    r = np.random.default_rng(1)
    x, dz = r.standard_normal((3, 2, 8)), r.standard_normal((3, 2, 8))
    w = r.standard_normal(8) if norm else None
    pos = r.integers(0, 1000, (3, len(pairs)))
    f = lambda x, w: OL.rope_fwd(x, w, pos, pairs, 100.0, 1e-3)
    dx, dw, _ = OL.rope_bwd(x, w, dz, pos, pairs, 100.0, 1e-3)
    np.testing.assert_allclose(dx, _difference(lambda t: f(t, w), x, dz), rtol=0, atol=1e-7)
    if norm:
        np.testing.assert_allclose(dw, _difference(lambda t: f(x, t), w, dz), rtol=0, atol=1e-7)


@pytest.mark.parametrize("window,n_sink", [(0, 0), (1, 0), (3, 2), (4, 20), (100, 1)])
def test_window_gradients(window, n_sink):
    r = np.random.default_rng(2)
    q, do = r.standard_normal((2, 9, 4, 4)), r.standard_normal((2, 9, 4, 4))
    k, v = r.standard_normal((2, 9, 2, 4)), r.standard_normal((2, 9, 2, 4))
    (dq, dk, dv), _ = OL.window_bwd(q, k, v, do, window, n_sink)
    f = lambda q, k, v: OL.window_fwd(q, k, v, window, n_sink)[0]
    for got, x, g in ((dq, q, lambda t: f(t, k, v)), (dk, k, lambda t: f(q, t, v)),
                      (dv, v, lambda t: f(q, k, t))):
        np.testing.assert_allclose(got, _difference(g, x, do), rtol=0, atol=1e-7)


def test_whole_window_is_causal_attention():
    r = np.random.default_rng(3)
    q, k, v = (r.standard_normal((2, 17, 3, 8)) for _ in range(3))
    ref = torch.nn.functional.scaled_dot_product_attention(
        *(torch.from_numpy(t).transpose(1, 2) for t in (q, k, v)), is_causal=True).transpose(1, 2)
    for window, n_sink in ((0, 0), (17, 0), (1, 17)):
        np.testing.assert_allclose(OL.window_fwd(q, k, v, window, n_sink)[0], ref.numpy(), atol=1e-12)


@pytest.mark.parametrize("window,n_sink", [(0, 0), (5, 2), (20, 3)])
def test_newest_token_is_the_last_row(window, n_sink):
    """A token over its pages sees what the last row of the windowed attention sees."""
    r = np.random.default_rng(4)
    L, page = 21, 16
    q, k, v = r.standard_normal((1, L, 4, 8)), r.standard_normal((1, L, 2, 8)), r.standard_normal((1, L, 2, 8))
    K, V = np.full((3, 2, page, 8), np.nan), np.full((3, 2, page, 8), np.nan)
    table = np.array([[2, 0]])
    K, V, qz = OL.paged_append(K, V, table, [L], [0, L], q[0], k[0], v[0], None, None, None, (), 10.0, 1e-6)
    out, _ = OL.paged_attn(qz[-1:], K, V, table, [L], window, n_sink)
    np.testing.assert_allclose(out[0], OL.window_fwd(q, k, v, window, n_sink)[0][0, -1], atol=1e-12)
