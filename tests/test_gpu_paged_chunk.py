"""Attention of the newest tokens of every sequence over the paged cache, in bf16 and quantised, against float64.
Bar: the probabilities are rounded to bf16 for their products (2^-8 of sum p |v|), the result once more (2^-8 of
itself), and the fp32 scores, exponentials and sums keep 2e-5 of sum p |v|.  What a quantised cache stands for is exact."""
import numpy as np
import pytest
import torch

import paper_2608_23463_gb300 as pf
from oracle import local as OL
from paper_2608_23463_gb300.local import PagedKVCache, QKRope, WindowAttention
from tests.test_gpu_local_rope import BF, check, f64, rand

pytestmark = pytest.mark.gpu
I8, I32 = torch.int8, torch.int32


def starts(new):
    return torch.tensor([0] + list(new)).cumsum(0).to(I32).cuda()


def make(length, H, KV, dh, page, seed, quant=False, spare=3, scale=1.0, **kw):
    """A cache whose sequences hold so many rows, in pages of any order."""
    B, need = len(length), [-(-n // page) for n in length]
    n_pages, most = sum(need) + spare, max(max(need), 1)
    rng = np.random.default_rng(seed)
    K, V = (scale * rng.standard_normal((n_pages, KV, page, dh)) for _ in range(2))
    if quant:
        (K, Ke), (V, Ve) = OL.quantise(K), OL.quantise(V)
        kw.update(dtype=I8, K_exp=torch.from_numpy(Ke).cuda(), V_exp=torch.from_numpy(Ve).cuda())
    K, V = (torch.from_numpy(t).to("cuda", I8 if quant else BF) for t in (K, V))
    table, order = np.full((B, most), -1, np.int32), rng.permutation(n_pages)
    for b, k in enumerate(need):
        table[b, :k], order = order[:k], order[k:]
    return PagedKVCache(B, H, KV, dh, page, n_pages, most, K=K, V=V, table=torch.from_numpy(table).cuda(),
                        len=torch.tensor(length, dtype=I32).cuda(), **kw)


def pools(c):
    """What the cache stands for, float64."""
    if c.dtype == I8:
        return tuple(OL.values(x.cpu().numpy(), e.cpu().numpy()) for x, e in ((c.K, c.K_exp), (c.V, c.V_exp)))
    return f64(c.K), f64(c.V)


def compare(c, q, start, out, rows=None):
    K, V = (np.nan_to_num(t, nan=0.0, posinf=0.0, neginf=0.0) for t in pools(c))
    s = start.tolist()
    ref, mag = OL.paged_chunk(f64(q).reshape(q.shape[0], -1, c.dh), K, V, np.maximum(c.table.cpu().numpy(), 0), c.len.tolist(), s,
                              c.desc.window, c.desc.n_sink)
    n = s[-1]
    rows = slice(0, n) if rows is None else rows
    ref, mag, got = ref[rows], mag[rows], f64(out).reshape(ref.shape)[rows]
    assert np.isfinite(got).all()
    err = np.abs(got - ref) - (2.0 ** -8 * 1.01 * (mag + np.abs(ref)) + 2e-5 * mag)
    assert (err <= 0).all(), (err.max(), np.argwhere(err > 0)[:5])


def chunk(c, new, seed, scale=1.5, pad=0):
    """One call, twice, against float64; rows of padding stay as they were."""
    start = starts(new)
    q = rand((sum(new) + pad, c.n_heads * c.dh), seed, scale=scale)
    out = torch.full_like(q, 7.0)
    c.attend(q, out=out, start=start)
    again = c.attend(q, start=start)
    check()
    n = sum(new)
    assert torch.equal(out[:n], again[:n]) and (out[n:] == 7).all()
    compare(c, q, start, out)
    return out


HEADS = [(1, 1, 64), (8, 2, 64), (16, 16, 128), (16, 1, 128), (9, 1, 64), (10, 2, 128), (24, 3, 64)]


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("H,KV,dh", HEADS)
@pytest.mark.parametrize("page,new,before", [
    (16, [1], [0]), (16, [1], [300]), (32, [3, 0, 1, 2], [0, 5, 127, 128]), (64, [130], [0]), (48, [7, 33, 1], [1000, 90, 0]),
    (128, [5, 0, 260], [256, 0, 13]), (16, [40, 1], [2500, 1])])
def test_lengths(quant, H, KV, dh, page, new, before):
    c = make([a + b for a, b in zip(new, before)], H, KV, dh, page, 1, quant)
    chunk(c, new, 2, pad=3 if len(new) > 1 else 0)


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("page,window,n_sink", [(144, 0, 0), (144, 300, 20), (256, 0, 0), (400, 150, 200), (80, 0, 0), (112, 500, 3),
                                                (1024, 0, 0)])
@pytest.mark.parametrize("KV,dh", [(2, 128), (4, 64)])
def test_pages_of_other_lengths(quant, page, window, n_sink, KV, dh):
    """Pages longer than a step, and such that neither fits the other."""
    new, before = [3, 1, 140, 1, 30], [1500, 2 * page, page - 70, page - 1, 897]
    c = make([a + b for a, b in zip(new, before)], 8, KV, dh, page, 60, quant, window=window, n_sink=n_sink)
    chunk(c, new, 61)


@pytest.mark.parametrize("quant", [False, True])
def test_sequences_that_share_pages(quant):
    """A prompt's pages in the tables of several sequences."""
    c = make([500, 480, 300], 8, 2, 64, 16, 62, quant, spare=0)
    c.table[1, :20] = c.table[0, :20]
    c.table[2, :18] = c.table[0, :18]
    c.len.copy_(torch.tensor([500, 480, 290], dtype=I32))
    chunk(c, [4, 120, 2], 63)


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("window,n_sink", [(1, 0), (1, 1), (5, 3), (16, 16), (64, 100), (1000, 2), (333, 17), (200, 3000),
                                           (129, (1 << 31) - 1), ((1 << 31) - 1, 5)])
@pytest.mark.parametrize("KV,dh,page", [(2, 128, 32), (8, 64, 16)])
def test_windows(quant, window, n_sink, KV, dh, page):
    """Pages that no token sees may be gone, and hidden rows hold anything."""
    new, before = [1, 0, 30, 150, 9], [16, 3, 333, 0, 1500]
    length = [a + b for a, b in zip(new, before)]
    c = make(length, 8, KV, dh, page, 3, quant, window=window, n_sink=n_sink)
    for b, n in enumerate(length):
        seen = np.zeros(n, bool)
        for i in range(n - new[b], n):
            seen |= OL.visible(i, n, window, n_sink)
        for p in range(-(-n // page)):
            rows = np.arange(p * page, (p + 1) * page)
            alive = np.array([r < n and seen[r] for r in rows])
            if not alive.any():
                c.table[b, p] = -7
                continue
            for r in rows[~alive] - p * page:  # past the end among them
                spoil(c, int(c.table[b, p]), slice(None), r)
    chunk(c, new, 4)


def spoil(c, page, head, row, value=float("nan")):
    if c.dtype == I8:
        c.K_exp[page, head, row] = c.V_exp[page, head, row] = -128
    else:
        c.K[page, head, row] = value
        c.V[page, head, row] = -value


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("before,new,window,sinks", [(0, 300, 0, 0), (700, 20, 0, 0), (2500, 3, 0, 0), (0, 300, 40, 3)])
def test_not_finite_beyond_a_token(quant, before, new, window, sinks):
    """A later token's row that is not finite reaches those that see it and no others; so too for a key head."""
    c = make([before + new], 8, 2, 64, 32, 5, quant, window=window, n_sink=sinks)
    start, q = starts([new]), rand((new, 512), 6)
    ref = c.attend(q, start=start)
    for i in (0, new // 2, new - 1):
        r = before + i
        saved = [t.clone() for t in (c.K, c.V)] + [t.clone() for t in (c.K_exp, c.V_exp) if quant]
        spoil(c, int(c.table[0, r // 32]), 1, r % 32, float("inf"))
        out = c.attend(q, start=start)
        check()
        seen = np.stack([OL.visible(before + t, before + new, window, sinks)[r] for t in range(new)])
        o, h = f64(out).reshape(new, 8, 64), f64(ref).reshape(new, 8, 64)
        assert (o[:, :4] == h[:, :4]).all()
        assert not np.isfinite(o[seen][:, 4:]).any()
        compare(c, q, start, torch.where(torch.isfinite(out), out, ref), np.flatnonzero(~seen))
        assert np.isfinite(o[~seen]).all()
        for t, s in zip((c.K, c.V) + ((c.K_exp, c.V_exp) if quant else ()), saved):
            t.copy_(s)


@pytest.mark.parametrize("dh,before,new", [(128, 0, 200), (64, 0, 100), (128, 3000, 5), (64, 3000, 5), (128, 1000, 300), (64, 6, 20)])
def test_one_column_not_finite_beyond_a_token(dh, before, new):
    """A hidden row with an infinity in one column alone: whole items, pieces of few items and of many."""
    c = make([before + new, 70], 8, 2, dh, 16, 64)
    r = before + new - 1
    for col in (0, 37, dh - 1):
        V = c.V.clone()
        c.V[int(c.table[0, r // 16]), 1, r % 16, col] = float("inf")
        start = starts([new, 3])
        q = rand((new + 3, 8 * dh), 65)
        out = c.attend(q, start=start)
        again = c.attend(q, start=start)
        check()
        assert torch.equal(out.view(torch.int16), again.view(torch.int16))
        sees = out[new - 1].view(8, dh)[4:]  # its own token's heads of that key head
        assert not sees[:, col].isfinite().any() and sees[:, [i for i in range(dh) if i != col]].isfinite().all()
        compare(c, q, start, torch.where(out.isfinite(), out, torch.zeros_like(out)), [i for i in range(new + 3) if i != new - 1])
        assert out[[i for i in range(new + 3) if i != new - 1]].isfinite().all()
        c.V.copy_(V)


def test_scores_far_apart():
    """Scores of hundreds (the reference is raised over and over), and all alike."""
    c = make([300, 77], 4, 2, 64, 16, 7)
    c.K.mul_(torch.linspace(0.1, 12, c.K.shape[2], device="cuda").to(BF)[:, None])
    chunk(c, [100, 77], 8, scale=8.0)
    c.K.fill_(-3.0)
    q = torch.full((30, 256), 64.0, dtype=BF, device="cuda")
    compare(c, q, starts([20, 10]), c.attend(q, start=starts([20, 10])))
    c.K.fill_(float("-inf"))  # every score -inf: 0 / 0
    out = c.attend(q, start=starts([20, 10]))
    check()
    assert out.isnan().all()


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("dh", [64, 128])
def test_pieces(quant, dh):
    """Few long caches, on many CTAs; many short ones, several to a CTA; and both."""
    c = make([9000], 4, 1, dh, 64, 9, quant)
    chunk(c, [2], 10)
    chunk(c, [70], 11)
    length = [(37 * i) % 90 + 8 for i in range(700)]
    c = make(length, 2, 2, dh, 16, 12, quant)
    chunk(c, [(5 * i) % 9 for i in range(700)], 13)
    length = [1 + (53 * i) % 190 for i in range(99)] + [6000]
    c = make(length, 8, 2, dh, 16, 14, quant)
    chunk(c, [min(n, 1 + i % 3) for i, n in enumerate(length)], 15)


@pytest.mark.parametrize("quant", [False, True])
def test_many_sequences(quant):
    """As many sequences as a call takes; and more than a warp's lanes share out at once."""
    for B, i0 in ((2048, 40), (129, 50)):
        length = [(29 * i) % 150 for i in range(B)]
        c = make(length, 2, 1, 64, 16, i0, quant)
        chunk(c, [min(n, (7 * i) % 4) for i, n in enumerate(length)], i0 + 1)


def test_many_items():
    """Enough items that none is cut: 4 * 16 heads of 33 pairs."""
    c = make([2100] * 4, 16, 16, 64, 64, 16)
    start, q = starts([2100] * 4), rand((8400, 1024), 17)
    out = c.attend(q, start=start)
    check()
    k, v = (t[c.table.long()].transpose(2, 3).reshape(4, -1, 16, 64)[:, :2100].reshape(8400, 1024) for t in (c.K, c.V))
    ref = WindowAttention(4, 2100, 16, 16).forward(q, k, v, train=False)
    check()
    # both round P and the result: twice the bar, with |p v| at most the largest value
    assert float((out.float() - ref.float()).abs().max()) <= 2 * 2 * 2.0 ** -8 * float(v.abs().max())
    some = [0, 1, 127, 128, 2099, 2100, 5000, 8399]  # and float64
    for r in some:
        b, i = divmod(r, 2100)
        o, mag = OL.window_fwd(*(f64(t.view(4, 2100, 16, 64)[b:b + 1, :i + 1]) if t is not q else
                                 f64(t.view(4, 2100, 16, 64)[b:b + 1, i:i + 1]).repeat(i + 1, 1) for t in (q, k, v)), 0, 0) \
            if i < 130 else (None, None)
        if o is not None:
            err = np.abs(f64(out[r]).reshape(16, 64) - o[0, -1])
            assert (err <= 2.0 ** -8 * 1.01 * (mag[0, -1] + np.abs(o[0, -1])) + 2e-5 * mag[0, -1]).all()


def test_prompts_then_tokens():
    """Prompts appended and attended in pieces, quantised and not, against one windowed call over the whole."""
    H, KV, dh, L = 8, 2, 64, 400
    x = rand((2 * L, (H + 2 * KV) * dh), 18)
    cut = lambda t: t.split((H * dh, KV * dh, KV * dh), 1)
    w = [1 + 0.1 * rand((dh,), s, torch.float32) for s in (19, 20)]
    rope = QKRope(H, KV, dh, *w)
    q, k, v = cut(x)
    ref = WindowAttention(2, L, H, KV, window=120, n_sink=4).forward(*rope.forward(q, k, L=L), v, train=False)
    for dtype in (BF, I8):
        c = PagedKVCache(2, H, KV, dh, 16, 60, 25, rope=rope, window=120, n_sink=4, dtype=dtype)
        c.reserve([L, L])
        got = [[], []]
        done = [0, 0]
        for n in ((100, 1), (0, 250), (200, 148), (99, 1), (1, 0)):
            rows = torch.cat([x[b * L + done[b]:b * L + done[b] + n[b]] for b in range(2)])
            s = starts(n)
            c.advance(s)
            o = c.attend(c.append(*cut(rows), start=s), start=s)
            got[0].append(o[:n[0]])
            got[1].append(o[n[0]:])
            done = [a + b for a, b in zip(done, n)]
        check()
        out = torch.cat(got[0] + got[1])
        bar = 4 * 2.0 ** -8 * float(v.abs().max()) if dtype == BF else 0.1
        assert out.shape == ref.shape and float((out.float() - ref.float()).abs().max()) <= bar


@pytest.mark.parametrize("quant", [False, True])
def test_rows_apart_and_streams(quant):
    c = make([40, 9, 500], 4, 2, 64, 16, 21, quant)
    start = starts([3, 0, 40])
    wide, out = rand((43, 4 * 256), 22), torch.full((43, 512), 7.0, dtype=BF, device="cuda")
    q = wide[:, 256:512]
    ref = c.attend(q.contiguous(), start=start)
    torch.cuda.synchronize()
    s = [torch.cuda.Stream() for _ in range(2)]
    outs = [out, out.clone()]
    torch.cuda.synchronize()
    for _ in range(10):
        for k in range(2):  # two calls of one cache at once
            with torch.cuda.stream(s[k]):
                c.attend(q, out=outs[k][:, 128:384], start=start)
    torch.cuda.synchronize()
    check()
    for o in outs:
        assert torch.equal(o[:, 128:384], ref) and (o[:, :128] == 7).all() and (o[:, 384:] == 7).all()


@pytest.mark.parametrize("quant", [False, True])
def test_long_cache_crosses_32_bits(quant):
    """A sequence whose pages lie past 2^32 values of the pool."""
    KV, dh, page, n_pages = 16, 128, 128, 16400
    K = torch.zeros((n_pages, KV, page, dh), dtype=I8 if quant else BF, device="cuda")
    c = PagedKVCache(1, KV, KV, dh, page, n_pages, 2, K=K, V=torch.zeros_like(K), dtype=K.dtype)
    c.table.copy_(torch.tensor([[n_pages - 1, n_pages - 2]], dtype=I32))
    x, s = rand((200, 3 * KV * dh), 23), starts([200])
    c.advance(s)
    q = c.append(*x.split(KV * dh, 1), start=s)
    out = c.attend(q, start=s)
    k, v = c.read(s, rows=200)
    check()
    assert not K[:2].any()
    ref, mag = OL.window_fwd(*(f64(t).reshape(1, 200, KV, dh) for t in (q, k, v)), 0, 0)
    err = np.abs(f64(out).reshape(ref.shape) - ref)
    assert (err <= 2.0 ** -8 * 1.01 * (mag + np.abs(ref)) + 2e-5 * mag).all()
    if not quant:
        assert torch.equal(k, x[:, KV * dh:2 * KV * dh]) and torch.equal(v, x[:, 2 * KV * dh:])


def test_what_cannot_be_is_flagged():
    c = make([20, 20, 20, 20], 2, 1, 64, 16, 24)
    q, start = rand((8, 128), 25), starts([2, 2, 2, 2])
    ref = c.attend(q, start=start)
    check()

    def flagged(start=start):
        out = c.attend(q, out=torch.full_like(q, 7.0), start=start)
        with pytest.raises(pf.ProxyFormerError) as e:
            check()
        assert e.value.status == pf.PF_ERR_CAPACITY
        return out
    length, table = c.len.clone(), c.table.clone()
    c.table[1, 1] = c.n_pages  # its second page: read as zeros
    out = flagged()
    assert torch.equal(out[:2], ref[:2]) and torch.equal(out[4:], ref[4:]) and out.isfinite().all()
    c.table.copy_(table)
    for bad in (1000, -1, 1, -(1 << 31), (1 << 31) - 1):
        c.len[2] = bad
        out = flagged()
        keep = [0, 1, 2, 3, 6, 7]
        assert torch.equal(out[keep], ref[keep]) and not out[4:6].any(), bad
    c.len.copy_(length)
    for bad in ([0, 2, 4, 6, 9], [-1, 2, 4, 6, 8], [0, 2, 1 << 30, 6, 8], [0, 2, 4, 6, -(1 << 31)], [3, 2, 4, 6, 8]):
        out = flagged(torch.tensor(bad, dtype=I32, device="cuda"))
        fine = [b for b in range(4) if 0 <= bad[b] <= bad[b + 1] <= 8 and bad[b] == 2 * b]
        for b in fine:
            if bad[b + 1] == 2 * b + 2:
                assert torch.equal(out[2 * b:2 * b + 2], ref[2 * b:2 * b + 2]), (bad, b)
    out = c.attend(q, start=start)
    check()
    assert torch.equal(out, ref)


@pytest.mark.parametrize("quant", [False, True])
def test_mixed_steps_in_a_graph(quant):
    """A captured step of as many rows serves other lengths and other chunks; two graphs share a cache."""
    c = make([1500, 700, 40], 4, 2, 64, 16, 26, quant)
    q, start = rand((24, 256), 27), starts([16, 1, 7])
    out = [torch.zeros_like(q) for _ in range(2)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.attend(q, out=out[0], start=start)
    torch.cuda.current_stream().wait_stream(s)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g, o in zip(graphs, out):
        with torch.cuda.graph(g, capture_error_mode="thread_local"):
            c.attend(q, out=o, start=start)
    for i, (new, length) in enumerate([([16, 1, 7], [1500, 700, 40]), ([0, 24, 0], [3, 700, 1]), ([1, 1, 1], [1, 1, 1]),
                                       ([2, 20, 2], [1400, 21, 39])]):
        q.copy_(rand((24, 256), 30 + i))
        start.copy_(starts(new))
        c.len.copy_(torch.tensor(length, dtype=I32))
        ref = c.attend(q, start=start)
        for o in out:
            o.fill_(7)
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        n = sum(new)
        for o in out:
            assert torch.equal(o[:n], ref[:n]) and (o[n:] == 7).all(), i
    check()


def test_no_tokens():
    c = make([20, 0], 2, 1, 64, 16, 28)
    assert c.attend(rand((0, 128), 29), start=starts([0, 0])).shape == (0, 128)
    q = rand((5, 128), 30)
    out = c.attend(q, out=torch.full_like(q, 7.0), start=starts([0, 0]))
    check()
    assert (out == 7).all()
