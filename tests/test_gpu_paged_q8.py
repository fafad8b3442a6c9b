"""The quantised paged cache against float64: rows as they are written and read back, and the newest token's attention
over them.  Whole numbers and exponents of values that come as they are (V, and K without norm and rotation) are the
definition's; normed and turned keys are quantised from fp32 values off by 4e-6 of their row's largest at most (fp32's
own bar of norm and rotation), so that each is within half a step of the definition's value and that much.  The
attention's bar is that of the bf16 cache, as what the rows stand for is exact."""
import numpy as np
import pytest
import torch

import paper_2608_23463_gb300 as pf
from oracle import local as OL
from paper_2608_23463_gb300.local import PagedKVCache, QKRope
from tests.test_gpu_local_rope import BF, EPS, F32, THETA, check, close, f64, rand, weights
from tests.test_gpu_paged_chunk import I8, I32, make, pools, spoil, starts

pytestmark = pytest.mark.gpu


def place(c, start):
    """Pages and rows of the call's tokens, start [batch + 1]."""
    n = c.len.tolist()
    b = np.repeat(np.arange(c.batch), np.diff(start))
    r = np.concatenate([np.arange(n[i] - (start[i + 1] - start[i]), n[i]) for i in range(c.batch)]).astype(int)
    return c.table.cpu().numpy()[b, r // c.page], r % c.page, r


@pytest.mark.parametrize("H,KV,dh,page,before,new,norm", [
    (1, 1, 64, 16, [0], None, True), (16, 16, 128, 64, [0, 1, 63, 64, 65, 127, 128, 1000], None, True),
    (10, 2, 64, 16, [0, 15, 31], [1, 40, 17], True), (4, 1, 128, 48, [7, 0, 47, 48, 200], [0, 300, 1, 0, 96], False),
    (6, 3, 64, 32, list(range(40)), [i % 3 for i in range(40)], True), (5, 5, 128, 16, [3, 900], [1200, 2], True)])
def test_append_and_read(H, KV, dh, page, before, new, norm):
    B = len(before)
    count = [1] * B if new is None else new
    rows = [a + b for a, b in zip(before, count)]
    w_q, w_k = weights(dh, 1) if norm else (None, None)
    rope = QKRope(H, KV, dh, w_q, w_k, theta=THETA, eps=EPS)
    c = make(before, H, KV, dh, page, 2, True, rope=rope, spare=sum(-(-r // page) for r in rows) + 2)
    # room for the new rows
    need, free = [-(-r // page) for r in rows], sorted(set(range(c.n_pages)) - set(c.table.flatten().tolist()))
    table = np.full((B, max(need)), -1, np.int32)
    for b, k in enumerate(need):
        own = [p for p in c.table[b].tolist() if p >= 0]
        table[b, :k] = own + [free.pop() for _ in range(k - len(own))]
    c = PagedKVCache(B, H, KV, dh, page, c.n_pages, max(need), rope=rope, K=c.K, V=c.V, K_exp=c.K_exp, V_exp=c.V_exp,
                     table=torch.from_numpy(table).cuda(), len=c.len, dtype=I8)
    was = [t.clone() for t in (c.K, c.V, c.K_exp, c.V_exp)]
    n = sum(count)
    x = rand((n, (H + 2 * KV) * dh + 8), 3, scale=1.5)
    q, k, v = x[:, :H * dh], x[:, H * dh:(H + KV) * dh], x[:, (H + KV) * dh:(H + 2 * KV) * dh]
    s = None if new is None else starts(new)
    c.advance(s)
    qz = c.append(q, k, v, start=s)
    ko, vo = c.read(s) if s is None else c.read(s, rows=n)
    check()
    pg, r, at = place(c, np.cumsum([0] + count))
    heads = lambda t: f64(t).reshape(n, KV, dh)
    close("q", qz, OL.rope_fwd(f64(q).reshape(n, H, dh), None if w_q is None else f64(w_q), at[:, None], (dh // 2,), THETA, EPS), BF)
    got = [t.cpu().numpy() for t in (c.K, c.V, c.K_exp, c.V_exp)]
    ref_x, ref_e = OL.quantise(heads(v))
    assert (got[1][pg, :, r] == ref_x).all() and (got[3][pg, :, r] == ref_e).all()
    y = OL.rope_fwd(heads(k), None if w_k is None else f64(w_k), at[:, None], (dh // 2,), THETA, EPS)
    kx, ke = got[0][pg, :, r], got[2][pg, :, r]
    val, size = OL.values(kx, ke), np.abs(y).max(-1, keepdims=True)
    step = np.ldexp(1.0, ke.astype(int))[..., None]
    assert (np.abs(val - y) <= 0.5 * step + 4e-6 * size).all()
    assert (size <= 127 * step * (1 + 1e-5)).all() and (size * (1 + 1e-5) > 127 * step / 2).all()  # the least power
    # what else the pools hold stays
    for a, b in zip(got, was):
        b = b.cpu().numpy()
        b[pg, :, r] = a[pg, :, r]
        assert (a == b).all()
    assert (heads(ko) == val).all() and (heads(vo) == OL.values(got[1][pg, :, r], got[3][pg, :, r])).all()


def test_rows_of_every_kind():
    """Ties, borders of the exponent, the least and largest values, zeros, and rows that are not finite; keys come as
    values without norm and rotation."""
    kinds = [np.full(64, 127.0), np.full(64, 127.5), np.full(64, 128.0), np.arange(64) / 2 + 95.5, np.zeros(64),
             np.full(64, 2.0 ** -133), np.full(64, 3 * 2.0 ** -127), np.full(64, 127 * 2.0 ** -126),
             np.full(64, 127 * 2.0 ** 104), np.full(64, 127.5 * 2.0 ** 104), np.full(64, 2.0 ** 127),
             np.r_[np.full(63, 1.0), np.inf], np.r_[-np.inf, np.zeros(63)], np.r_[np.nan, np.full(63, 5.0)],
             np.r_[127 * 2.0 ** 104, np.full(63, -1.0)], -np.arange(64) * 1.5, np.r_[np.full(32, 0.5), np.full(32, -0.5), ] * 127,
             np.r_[1e-30, np.full(63, 1e-33)], np.full(64, -63.5), np.full(64, 63.75)]
    x = torch.tensor(np.array(kinds), dtype=F32).to("cuda", BF)
    n = len(kinds)
    c = PagedKVCache(1, 1, 1, 64, 16, 4, 3, dtype=I8)
    c.reserve([n])
    s = starts([n])
    c.advance(s)
    c.append(None, x, x.flip(0), start=s)
    k, v = c.read(s, rows=n)
    check()
    pg, r, _ = place(c, [0, n])
    for t, e, y, back in ((c.K, c.K_exp, x, k), (c.V, c.V_exp, x.flip(0), v)):
        ref_x, ref_e = OL.quantise(f64(y))
        fine = ref_e != -128
        got_e = e.cpu().numpy()[pg, 0, r]
        assert (got_e == ref_e).all()
        assert (t.cpu().numpy()[pg, 0, r][fine] == ref_x[fine]).all()
        np.testing.assert_array_equal(f64(back), OL.values(ref_x, ref_e))


@pytest.mark.parametrize("KV,dh,page", [(1, 64, 16), (3, 128, 48), (16, 128, 64), (40, 64, 16)])
def test_read_of_both_caches(KV, dh, page):
    """Whole caches and the newest rows, into columns of wider matrices, rows behind the last sequence left alone."""
    length = [100, 0, 1, 333, 16]
    for quant in (False, True):
        c = make(length, KV, KV, dh, page, 5, quant)
        s = starts(length)
        out = [torch.full((455, 2 * KV * dh), 7.0, dtype=BF, device="cuda") for _ in range(2)]
        c.read(s, out=[t[:, KV * dh:] for t in out])
        pg, r, _ = place(c, s.tolist())
        newest = c.read(starts([1, 0, 1, 1, 1]), rows=4)
        check()
        for t, last, pool in zip(out, newest, pools(c)):
            assert (t[:, :KV * dh] == 7).all() and (t[450:] == 7).all()
            got, ref = f64(t[:450, KV * dh:]), pool[pg, :, r].reshape(450, -1)
            assert (got == ref).all() and (f64(last) == ref[[99, 100, 433, 449]]).all()
        if 0 in length:  # one row of each, though one has none
            k, v = c.read()
            with pytest.raises(pf.ProxyFormerError) as e:
                check()
            assert e.value.status == pf.PF_ERR_CAPACITY
            assert torch.equal(k[[0, 2, 3, 4]], newest[0]) and not k[1].any() and not v[1].any()


def test_read_flags():
    for quant in (False, True):
        c = make([20, 20], 2, 1, 64, 16, 6, quant)
        s = starts([20, 20])
        ref = c.read(s, rows=40)[0]
        check()
        c.table[0, 1], c.len[1] = c.n_pages + 5, 7
        k, _ = c.read(s, rows=40)
        with pytest.raises(pf.ProxyFormerError) as e:
            check()
        assert e.value.status == pf.PF_ERR_CAPACITY
        assert torch.equal(k[:16], ref[:16]) and not k[16:33].any() and torch.equal(k[33:], ref[20:27])
        c.len[1] = 1000
        assert not c.read(s, rows=40)[0][20:].any()
        with pytest.raises(pf.ProxyFormerError):
            check()


def attend(c, q):
    out = c.attend(q)
    again = c.attend(q)
    check()
    assert torch.equal(out, again)
    K, V = (np.nan_to_num(t) for t in pools(c))
    ref, mag = OL.paged_attn(f64(q).reshape(c.batch, -1, c.dh), K, V, f64(c.table).astype(int), c.len.tolist(),
                             c.desc.window, c.desc.n_sink)
    err = np.abs(f64(out).reshape(ref.shape) - ref)
    assert (err <= 2.0 ** -8 * 1.01 * (mag + np.abs(ref)) + 2e-5 * mag).all(), (err - 2.0 ** -8 * (mag + np.abs(ref))).max()
    return out


@pytest.mark.parametrize("H,KV,dh", [(1, 1, 64), (8, 2, 64), (16, 16, 128), (16, 1, 128), (9, 1, 64), (10, 2, 128),
                                     (24, 3, 64)])
@pytest.mark.parametrize("page,length", [(16, [0, 1, 15, 16, 17, 63, 64, 65]), (48, [1000, 0, 3, 129, 0]), (64, [513]),
                                         (16, [4100, 1, 700])])
def test_lengths(H, KV, dh, page, length):
    c = make(length, H, KV, dh, page, 7, True)
    attend(c, rand((len(length), H * dh), 8, scale=1.5))


@pytest.mark.parametrize("window,n_sink", [(1, 0), (5, 3), (16, 16), (64, 100), (1000, 2), (700, 5000), (333, 17)])
@pytest.mark.parametrize("KV,dh", [(2, 128), (4, 64)])
def test_windows(window, n_sink, KV, dh):
    length = [0, 1, 16, 17, 100, 333, 1999, 2048]
    c = make(length, 8, KV, dh, 32, 9, True, window=window, n_sink=n_sink)
    for b, n in enumerate(length):
        seen = OL.visible(n - 1, n, window, n_sink) if n else np.zeros(0, bool)
        for p in range(-(-n // 32)):
            alive = [r < n and seen[r] for r in range(p * 32, p * 32 + 32)]
            if not any(alive):
                c.table[b, p] = -7
            else:
                for r in np.flatnonzero(~np.array(alive)):  # past the end among them
                    spoil(c, int(c.table[b, p]), slice(None), r)
    attend(c, rand((8, 8 * dh), 10))


def test_values_far_apart():
    """Rows whose powers of two lie far apart, in keys and in values; a row that is not finite."""
    c = make([300, 77], 4, 2, 64, 16, 11, True)
    c.V_exp.add_(torch.randint(-30, 30, c.V_exp.shape, generator=torch.Generator().manual_seed(1)).to("cuda", I8))
    attend(c, rand((2, 256), 12))
    c.K_exp.add_(torch.randint(-3, 5, c.K_exp.shape, generator=torch.Generator().manual_seed(2)).to("cuda", I8))
    ref = attend(c, rand((2, 256), 13, scale=4.0))
    pg = int(c.table[0, 3])
    c.V_exp[pg, 1, 5] = -128
    out = c.attend(rand((2, 256), 13, scale=4.0))
    check()
    assert out[0, 128:].isnan().all() and torch.equal(out[0, :128], ref[0, :128]) and torch.equal(out[1], ref[1])


@pytest.mark.parametrize("B,H,KV,dh,longest", [(160, 4, 2, 64, 2100), (40, 8, 4, 64, 2000), (38, 4, 4, 128, 400)])
def test_pairs_and_splits(B, H, KV, dh, longest):
    length = [0, 0] + [(53 * i) % 190 for i in range(B - 3)] + [longest]
    c = make(length, H, KV, dh, 16, 14, True)
    attend(c, rand((B, H * dh), 15))


def test_steps_in_a_graph():
    """Advance, append, attend and read of a quantised cache as one captured step, beside the same without a graph."""
    rope = QKRope(4, 2, 64, *(torch.ones(64, device="cuda") for _ in range(2)))
    c, e = (PagedKVCache(2, 4, 2, 64, 16, 10, 5, rope=rope, window=20, n_sink=2, dtype=I8) for _ in range(2))
    for t in (c, e):
        t.reserve([80, 80])
    buf = rand((2, 512), 16)
    mk = lambda: [torch.empty((2, 256), dtype=BF, device="cuda")] + [torch.empty((2, 128), dtype=BF, device="cuda") for _ in range(2)]
    out, ref = mk(), mk()

    def step(t, x, o):
        t.advance()
        t.attend(t.append(x[:, :256], x[:, 256:384], x[:, 384:]), out=o[0])
        t.read(out=o[1:])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(c, buf, out)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, capture_error_mode="thread_local"):
        step(c, buf, out)
    step(e, buf, ref)
    for i in range(40):
        x = rand((2, 512), 20 + i)
        buf.copy_(x)
        g.replay()
        step(e, x, ref)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, ref)), i
    check()
    assert c.len.tolist() == [41, 41]
