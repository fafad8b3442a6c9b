"""Norm and rotation of queries and keys, alone and on the way into the paged cache,
against float64.  Bars: results in bf16 are rounded once (2^-8 relative) from fp32
values, whose own error (norm over up to 128 values, sines to 2^-20, products) stays
below 1e-5 of the turned pair; fp32 results keep 4e-6 of it."""
import numpy as np
import pytest
import torch

import paper_2608_23463_gb300 as pf
from oracle import local as OL
from paper_2608_23463_gb300.local import PagedKVCache, QKRope

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
THETA, EPS = 10000.0, 1e-6


def rand(shape, seed, dtype=BF, scale=1.0):
    t = torch.from_numpy(np.random.default_rng(seed).standard_normal(shape).astype(np.float32) * scale)
    return t.to("cuda", dtype)


def f64(t):
    return t.detach().to("cpu", torch.float64).numpy()


def weights(dh, seed):
    return 1.0 + 0.3 * rand((dh,), seed, F32), 1.0 + 0.3 * rand((dh,), seed + 1, F32)


def check():
    pf.pf_sync_check(torch.cuda.current_stream().cuda_stream)


def close(name, got, ref, dtype, size=None):
    """|got - ref| within its rounding and the fp32 arithmetic's share of `size` (default: the head's largest)."""
    got = f64(got).reshape(ref.shape)
    size = np.abs(ref).max(-1, keepdims=True) if size is None else size
    bar = 2.0 ** -8 * 1.01 * np.abs(ref) + 1e-5 * size if dtype == BF else 4e-6 * size
    worst = (np.abs(got - ref) - bar).max() if ref.size else 0.0
    assert np.isfinite(got).all() and worst <= 0, f"{name}: {worst:.3e} above its bar"


def positions(rows, axes, seed, top):
    if axes == 0:
        return None
    return torch.from_numpy(np.random.default_rng(seed).integers(0, top, (rows, axes)).astype(np.int32)).cuda()


CASES = [  # rows, L, heads, kv, dh, pairs, norm, pos top (0: the row), dtype
    (1, 1, 1, 1, 64, (32,), True, 0, BF), (66, 33, 8, 2, 64, (32,), True, 0, BF),
    (37, 37, 5, 5, 128, (64,), True, 1 << 20, BF), (130, 65, 16, 1, 64, (16, 16), True, 512, BF),
    (9, 9, 3, 3, 128, (22, 21, 21), True, 100, F32), (70, 70, 6, 2, 64, (32,), True, 0x7fffffff, F32),
    (5000, 5000, 7, 1, 64, (20,), True, 0, BF), (50, 50, 4, 4, 128, (), True, 0, BF),
    (51, 17, 4, 2, 64, (32,), False, 0, BF), (33, 33, 32, 8, 128, (0, 64), False, 1 << 30, F32)]


@pytest.mark.parametrize("case", CASES)
def test_rope(case):
    rows, L, H, KV, dh, pairs, norm, top, dt = case
    # columns of a wider matrix, as a projection leaves them
    x, g = (rand((rows, (H + 2 * KV) * dh + 16), s, dt, 2.0) for s in (1, 2))
    cut = lambda t: (t[:, :H * dh], t[:, H * dh:(H + KV) * dh])
    w_q, w_k = weights(dh, 3) if norm else (None, None)
    op = QKRope(H, KV, dh, w_q, w_k, pairs=pairs, theta=THETA, eps=EPS, dtype=dt)
    pos = positions(rows, len(pairs), 5, top) if top else None
    at = np.arange(rows)[:, None] % L if pos is None else f64(pos)
    if not pairs:
        at = np.zeros((rows, 0))
    kw = dict(L=L, pos=pos)
    z = op.forward(*cut(x), **kw)
    d = op.backward(*cut(x), *cut(g), **kw)
    again = op.backward(*cut(x), *cut(g), **kw)
    check()
    for a, b in zip(d, again):
        assert a is b is None or torch.equal(a, b)
    for i, (n, w) in enumerate((("q", w_q), ("k", w_k))):
        xr = f64(cut(x)[i]).reshape(rows, -1, dh)
        gr = f64(cut(g)[i]).reshape(rows, -1, dh)
        wr = None if w is None else f64(w)
        close(n, z[i], OL.rope_fwd(xr, wr, at, pairs, THETA, EPS), dt)
        dx, dw, mag = OL.rope_bwd(xr, wr, gr, at, pairs, THETA, EPS)
        r = 1.0 if w is None else 1.0 / np.sqrt(np.mean(xr * xr, -1, keepdims=True) + EPS)
        close("d" + n, d[i], dx, dt, 2 * r * np.abs(gr).max(-1, keepdims=True) * (1 if w is None else np.abs(wr).max()))
        if w is None:
            assert d[2 + i] is None
        else:  # fp32 sums of at most a few hundred terms a lane: 2^-24 each, and the terms' own 4e-6
            assert (np.abs(f64(d[2 + i]) - dw) <= 4e-5 * mag + 1e-12).all()


def test_rope_in_place_and_one_sided():
    """Results over the inputs; a norm of the queries alone; a weight's gradient not asked for."""
    q, k, dq, dk = rand((40, 256), 1), rand((40, 128), 2), rand((40, 256), 3), rand((40, 128), 4)
    w_q, _ = weights(64, 5)
    op = QKRope(4, 2, 64, w_q, None)
    z, d = op.forward(q, k), op.backward(q, k, dq, dk)
    dq2, dk2, q2, k2 = dq.clone(), dk.clone(), q.clone(), k.clone()
    assert op.forward(q2, k2, out=(q2, k2))[0] is q2
    e = op.backward(q, k, dq2, dk2, out=(dq2, dk2))
    check()
    assert d[3] is None and torch.equal(e[2], d[2])
    for a, b in ((q2, z[0]), (k2, z[1]), (dq2, d[0]), (dk2, d[1])):
        assert torch.equal(a, b)


def test_rope_differences():
    """The gradient against differences of the forward in fp32: a step of 2^-6 leaves its
    square's share (2^-12 of curvature of order 1) and 1e-6 / 2^-6 of rounding."""
    q, k, dq, dk = (rand((3, 64), s, F32) for s in (1, 2, 3, 4))
    w_q, w_k = weights(64, 5)
    op = QKRope(1, 1, 64, w_q, w_k, dtype=F32)
    d = op.backward(q, k, dq, dk)
    step = 2.0 ** -6
    for c in (0, 1, 17, 63):
        e = torch.zeros_like(q)
        e[:, c] = step
        up, dn = op.forward(q + e, k + e), op.forward(q - e, k - e)
        for i, g in enumerate((dq, dk)):
            diff = ((up[i] - dn[i]).double() * g.double()).sum(1) / (2 * step)
            assert (diff - d[i][:, c].double()).abs().max() <= 64 * 2.0 ** -12 + 64 * 1e-6 / step


def test_rope_empty_and_zero_rows():
    w_q, w_k = weights(64, 5)
    op = QKRope(2, 1, 64, w_q, w_k)
    e = lambda n: torch.empty((0, n), dtype=BF, device="cuda")
    assert op.forward(e(128), e(64))[0].shape == (0, 128)
    d = op.backward(e(128), e(64), e(128), e(64))
    assert not d[2].any() and not d[3].any()
    z = torch.zeros((3, 128), dtype=BF, device="cuda")  # a zero row's norm is 1 / sqrt(eps)
    out = op.forward(z, z[:, :64])
    check()
    assert not out[0].any() and not out[1].any()


def test_rope_on_another_stream():
    q, k = rand((500, 512), 1), rand((500, 128), 2)
    op = QKRope(8, 2, 64)
    ref = op.forward(q, k)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        q2 = q * 1
        out = op.forward(q2, k)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, ref))


def paged(B, H, KV, dh, page, length, seed, rope=None, spare=3, **kw):
    """A cache whose sequences hold length[b] rows on pages in random order, the rest of the pool NaN."""
    rng = np.random.default_rng(seed)
    need = [-(-int(n) // page) for n in length]
    order = rng.permutation(sum(need) + spare)
    table = np.full((B, max(max(need), 1) + 1), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    n_pages = len(order)
    K, V = (np.full((n_pages, KV, page, dh), np.nan, np.float32) for _ in range(2))
    for b, n in enumerate(length):
        j = np.arange(n)
        for t in (K, V):
            t[table[b, j // page], :, j % page] = rng.standard_normal((int(n), KV, dh))
    dev = lambda a, d: torch.from_numpy(a).to("cuda", d)
    return PagedKVCache(B, H, KV, dh, page, n_pages, table.shape[1], rope=rope, K=dev(K, BF), V=dev(V, BF),
                        table=dev(table, torch.int32), len=dev(np.asarray(length, np.int32), torch.int32), **kw)


@pytest.mark.parametrize("B,H,KV,dh,page,before,new,norm", [
    (1, 1, 1, 64, 16, [0], None, True), (8, 16, 16, 128, 64, [0, 1, 63, 64, 65, 127, 128, 1000], None, True),
    (3, 10, 2, 64, 16, [0, 15, 31], [1, 40, 17], True), (5, 4, 1, 128, 48, [7, 0, 47, 48, 200], [0, 300, 1, 0, 96], False),
    (40, 6, 3, 64, 32, list(range(40)), [i % 3 for i in range(40)], True)])
def test_append(B, H, KV, dh, page, before, new, norm):
    start = None if new is None else np.concatenate([[0], np.cumsum(new)])
    new = [1] * B if new is None else new
    w_q, w_k = weights(dh, 3) if norm else (None, None)
    rope = QKRope(H, KV, dh, w_q, w_k, theta=THETA, eps=EPS)
    total = [a + b for a, b in zip(before, new)]
    c = paged(B, H, KV, dh, page, total, 7, rope)
    c.len.copy_(torch.tensor(before, dtype=torch.int32))
    n = sum(new)
    x = rand((n, (H + 2 * KV) * dh), 8, scale=2.0)
    q, k, v = x[:, :H * dh], x[:, H * dh:(H + KV) * dh], x[:, (H + KV) * dh:]
    K0, V0 = f64(c.K), f64(c.V)
    s = None if start is None else torch.from_numpy(start.astype(np.int32)).cuda()
    c.advance(s)
    qo = c.append(q, k, v, start=s)
    check()
    assert c.len.tolist() == total
    split = lambda t: f64(t).reshape(n, -1, dh)
    ws = [None if w is None else f64(w) for w in (w_q, w_k)]
    K, V, qz = OL.paged_append(K0, V0, f64(c.table).astype(int), total, np.arange(B + 1) if start is None else start,
                               split(q), split(k), split(v), *ws, None, (dh // 2,), THETA, EPS)
    close("q", qo, qz, BF)
    np.testing.assert_array_equal(f64(c.V), V)  # values are copied, nothing else is touched
    held = np.isfinite(K)
    assert (np.isfinite(f64(c.K)) == held).all()
    close("K", torch.from_numpy(np.where(held, f64(c.K), 0)), np.where(held, K, 0), BF)
    # keys alone, at given positions
    pos = positions(n, 1, 9, 1 << 24)
    assert c.append(None, k, v, start=s, pos=pos) is None
    check()
    K, _, _ = OL.paged_append(K0, V0, f64(c.table).astype(int), total, np.arange(B + 1) if start is None else start,
                              split(q), split(k), split(v), *ws, f64(pos), (dh // 2,), THETA, EPS)
    close("K at pos", torch.from_numpy(np.where(held, f64(c.K), 0)), np.where(held, K, 0), BF)


def test_append_out_of_range_is_flagged_and_left_out():
    c = paged(4, 2, 1, 64, 16, [16, 16, 16, 16], 1)
    c.len.copy_(torch.tensor([16, 33, 0, 17], dtype=torch.int32))  # full; past the table; no row; no page
    K0 = c.K.clone()
    x = rand((4, 256), 2)
    qo = c.append(x[:, :128], x[:, 128:192], x[:, 192:])
    with pytest.raises(pf.ProxyFormerError) as e:
        check()
    assert e.value.status == pf.PF_ERR_CAPACITY
    assert torch.equal(qo, x[:, :128])
    pg = int(c.table[0, 0])
    assert torch.equal(c.K[pg, 0, 15], x[0, 128:192])
    c.K[pg, 0, 15] = K0[pg, 0, 15]
    assert torch.equal(torch.nan_to_num(c.K), torch.nan_to_num(K0))
    c.len.copy_(torch.tensor([31, 32, -1, 5], dtype=torch.int32))
    c.advance()
    with pytest.raises(pf.ProxyFormerError):
        check()
    assert c.len.tolist() == [32, 32, -1, 6]
    check()  # the flag was cleared


def test_pages_are_reserved_and_released():
    c = PagedKVCache(2, 2, 1, 64, 16, n_pages=4, max_pages=3)
    c.reserve([17, 5])
    assert len({p for h in c.held for p in h}) == 3 and (c.table >= 0).sum() == 3
    c.reserve([32, 16])
    assert (c.table >= 0).sum() == 3
    with pytest.raises(pf.ProxyFormerError) as e:
        c.reserve([32, 33])
    assert e.value.status == pf.PF_ERR_CAPACITY
    c.release(0)
    c.reserve([0, 48])
    assert len(c.free) == 1 and len(c.held[1]) == 3


def test_released_sequences_write_nowhere():
    """A released sequence's token in a step of one for all is flagged, and the pages' next owner keeps its rows."""
    c = PagedKVCache(2, 2, 1, 64, 16, n_pages=4, max_pages=3)
    starts = lambda *s: torch.tensor(s, dtype=torch.int32, device="cuda")
    cut = lambda x: (x[:, :128], x[:, 128:192], x[:, 192:])
    c.reserve([20, 0])
    c.advance(starts(0, 20, 20))
    c.append(*cut(rand((20, 256), 1)), start=starts(0, 20, 20))
    c.release(0)
    c.reserve([0, 40])
    c.advance(starts(0, 0, 30))
    c.append(*cut(rand((30, 256), 2)), start=starts(0, 0, 30))
    check()
    rows = lambda: [t[c.table[1, :3].long()].transpose(1, 2).reshape(48, 64).clone() for t in (c.K, c.V)]
    before, x = rows(), rand((2, 256), 3)
    c.advance()
    c.append(*cut(x))  # a token for the released sequence too
    with pytest.raises(pf.ProxyFormerError) as e:
        check()
    assert e.value.status == pf.PF_ERR_CAPACITY
    for a, b, new in zip(rows(), before, cut(x)[1:]):
        b[30] = new[1]
        assert torch.equal(a, b)
    c.reserve([16, 40])
    assert c.len.tolist() == [0, 31]


@pytest.mark.parametrize("theta,pairs", [(0.1, (32,)), (1e-3, (32,)), (0.01, (12, 20)), (1e-5, (1, 2, 3))])
def test_small_theta(theta, pairs):
    """Frequencies of more than a turn a position."""
    op = QKRope(2, 1, 64, pairs=pairs, theta=theta, dtype=F32)
    pos = np.random.default_rng(1).integers(0, 1000, (200, len(pairs)))
    q, k = rand((200, 128), 2, F32), rand((200, 64), 3, F32)
    z = op.forward(q, k, pos=torch.from_numpy(pos.astype(np.int32)).cuda())
    check()
    for a, b in zip(z, (q, k)):
        close("turned", a, OL.rope_fwd(f64(b).reshape(200, -1, 64), None, pos, pairs, theta, 1e-6), F32)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_eps_below_fp32(dtype):
    """An epsilon that fp32 does not hold: rows of zeros stay zeros."""
    op = QKRope(2, 1, 64, *weights(64, 5), eps=1e-60, dtype=dtype)
    q, k = rand((4, 128), 1, dtype), rand((4, 64), 2, dtype)
    q[2], k[1] = 0, 0
    z = op.forward(q, k)
    check()
    for a, b, w in zip(z, (q, k), (op.w_q, op.w_k)):
        close("normed", a, OL.rope_fwd(f64(b).reshape(4, -1, 64), f64(w), np.arange(4)[:, None], (32,), 1e4, 1e-60), dtype)
