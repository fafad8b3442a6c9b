"""Attention of the newest token over the paged cache against float64.  Bar: the
probabilities are rounded to bf16 for their products (2^-8 of sum p |v|), the
result once more (2^-8 of itself), and the fp32 scores, exponentials and sums keep
2e-5 of sum p |v|."""
import math

import numpy as np
import pytest
import torch

import paper_2608_23463_gb300 as pf
from oracle import local as OL
from tests.test_gpu_local_rope import BF, check, f64, paged, rand

pytestmark = pytest.mark.gpu


def attend(c, q, scale=1.0):
    out = c.attend(q)
    again = c.attend(q)
    check()
    assert torch.equal(out, again)
    B, dh = c.batch, c.dh
    K, V = (np.nan_to_num(f64(t)) for t in (c.K, c.V))
    ref, mag = OL.paged_attn(f64(q).reshape(B, -1, dh), K, V, f64(c.table).astype(int), c.len.tolist(),
                             c.desc.window, c.desc.n_sink)
    err = np.abs(f64(out).reshape(ref.shape) - ref)
    assert (err <= 2.0 ** -8 * 1.01 * (mag + np.abs(ref)) + 2e-5 * mag).all(), (err - 2.0 ** -8 * (mag + np.abs(ref))).max()
    return out


@pytest.mark.parametrize("H,KV,dh", [(1, 1, 64), (8, 2, 64), (16, 16, 128), (16, 1, 128), (9, 1, 64), (10, 2, 128),
                                     (24, 3, 64)])
@pytest.mark.parametrize("page,length", [(16, [0, 1, 15, 16, 17, 63, 64, 65]), (48, [1000, 0, 3, 129, 0]), (64, [513]),
                                         (128, [0]), (16, [4100, 1, 700])])
def test_lengths(H, KV, dh, page, length):
    c = paged(len(length), H, KV, dh, page, length, 1)
    attend(c, rand((len(length), H * dh), 2, scale=1.5))


@pytest.mark.parametrize("window,n_sink", [(1, 0), (1, 1), (5, 3), (16, 16), (17, 4), (64, 100), (1000, 2), (700, 5000),
                                           (333, 17)])
@pytest.mark.parametrize("KV,dh", [(2, 128), (4, 64)])
def test_windows(window, n_sink, KV, dh):
    length = [0, 1, 16, 17, 100, 333, 1999, 2048]
    c = paged(8, 8, KV, dh, 32, length, 3, window=window, n_sink=n_sink)
    # pages that no token sees may hold anything, or be gone
    for b, n in enumerate(length):
        j = np.flatnonzero(~OL.visible(n - 1, n, window, n_sink)) if n else np.zeros(0, int)
        seen = {i // 32 for i in range(n) if i not in set(j.tolist())}
        for p in range(-(-n // 32)):
            if p not in seen:
                c.table[b, p] = -7
        for i in j.tolist():  # hidden rows of pages that are seen
            if i // 32 in seen:
                c.K[int(c.table[b, i // 32]), :, i % 32] = float("nan")
                c.V[int(c.table[b, i // 32]), :, i % 32] = float("inf")
    attend(c, rand((8, 8 * dh), 4))


def test_scores_far_apart():
    """Scores of hundreds (the reference is raised over and over) and of the lowest values."""
    c = paged(2, 4, 2, 64, 16, [300, 77], 5)
    c.K.mul_(torch.linspace(0.1, 12, c.K.shape[2], device="cuda").to(BF)[:, None])
    attend(c, rand((2, 256), 6, scale=8.0))
    c.K.fill_(-3.0)  # every score the same, -8 * 3 * 64
    q = torch.full((2, 256), 64.0, dtype=BF, device="cuda")
    attend(c, q)


def test_rows_apart_and_streams():
    c = paged(3, 4, 2, 64, 16, [40, 0, 200], 7)
    wide, out = rand((3, 4 * 256), 8), torch.full((3, 512), 7.0, dtype=BF, device="cuda")
    q = wide[:, 256:512]
    ref = c.attend(q.contiguous())
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c.attend(q * 1, out=out[:, 128:384])
    s.synchronize()
    check()
    assert torch.equal(out[:, 128:384], ref) and (out[:, :128] == 7).all() and (out[:, 384:] == 7).all()


def test_many_sequences():
    length = [(37 * i) % 150 for i in range(700)]
    c = paged(700, 2, 2, 64, 16, length, 9)
    attend(c, rand((700, 128), 10))


def test_long_cache_crosses_32_bits():
    """One sequence whose pages lie past 2^32 elements of the pool."""
    KV, dh, page, n_pages = 16, 128, 128, 16400  # 4.3e9 elements a pool
    assert n_pages * KV * page * dh > 1 << 32
    K = torch.zeros((n_pages, KV, page, dh), dtype=BF, device="cuda")
    V = torch.zeros_like(K)
    from paper_2608_23463_gb300.local import PagedKVCache
    c = PagedKVCache(1, KV, KV, dh, page, n_pages, 2, K=K, V=V)
    c.table.copy_(torch.tensor([[n_pages - 1, n_pages - 2]], dtype=torch.int32))
    x = rand((200, 3 * KV * dh), 11)
    s = torch.tensor([0, 200], dtype=torch.int32, device="cuda")
    c.advance(s)
    q = c.append(*x.split(KV * dh, 1), start=s)[-1:].contiguous()
    out = c.attend(q)
    check()
    assert torch.equal(q, x[-1:, :KV * dh]) and not K[:2].any()
    k, v = (f64(t).reshape(200, KV, dh) for t in x.split(KV * dh, 1)[1:])
    ref, mag = OL.window_fwd(f64(x[:, :KV * dh]).reshape(1, 200, KV, dh)[:, -1:].repeat(200, 1), k[None], v[None], 0, 0)
    err = np.abs(f64(out).reshape(KV, dh) - ref[0, -1])
    assert (err <= 2.0 ** -8 * 1.01 * (mag[0, -1] + np.abs(ref[0, -1])) + 2e-5 * mag[0, -1]).all()


def test_bad_pages_and_lengths_are_flagged():
    c = paged(3, 2, 1, 64, 16, [20, 20, 20], 12)
    q = rand((3, 128), 13)
    ref = c.attend(q)
    c.table[1, 1] = c.n_pages
    c.len[2] = 1000
    out = c.attend(q)
    with pytest.raises(pf.ProxyFormerError) as e:
        check()
    assert e.value.status == pf.PF_ERR_CAPACITY
    assert torch.equal(out[0], ref[0]) and not out[2].any() and torch.isfinite(out).all()


def test_decode_step_in_a_graph():
    """The lengths live on the device: a captured step (advance, append, attend) serves all the next ones."""
    from paper_2608_23463_gb300.local import PagedKVCache, QKRope
    rope = QKRope(4, 2, 64, *(torch.ones(64, device="cuda") for _ in range(2)))
    c, e = (PagedKVCache(2, 4, 2, 64, 16, 10, 5, rope=rope, window=20, n_sink=2) for _ in range(2))
    for t in (c, e):
        t.reserve([80, 80])
    x = rand((2, 512), 14)
    out = torch.empty((2, 256), dtype=BF, device="cuda")

    def step(t, x, out):
        t.advance()
        t.attend(t.append(x[:, :256], x[:, 256:384], x[:, 384:]), out=out)
    buf = x.clone()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step(c, buf, out)  # outside the graph once
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, capture_error_mode="thread_local"):
        step(c, buf, out)
    ref = torch.empty_like(out)
    step(e, x, ref)
    for i in range(40):
        xi = rand((2, 512), 20 + i)
        buf.copy_(xi)
        g.replay()
        step(e, xi, ref)
        torch.cuda.synchronize()
        assert torch.equal(out, ref), i
    check()
    assert c.len.tolist() == [41, 41]


@pytest.mark.parametrize("B,H,KV,dh,longest", [(160, 4, 2, 64, 2100), (40, 24, 8, 128, 2500), (400, 1, 1, 64, 5000),
                                               (40, 8, 4, 64, 2000), (38, 4, 4, 128, 400), (3, 8, 2, 64, 384), (3, 8, 2, 64, 385)])
def test_pairs_and_splits(B, H, KV, dh, longest):
    """More (sequence, key head) pairs than CTAs with long and empty ones among them, and either side of where a CTA
    takes a whole pair."""
    length = [0, 0] + [(53 * i) % 190 for i in range(B - 3)] + [longest]
    c = paged(B, H, KV, dh, 16, length, 11)
    attend(c, rand((B, H * dh), 12))
    c = paged(B, H, KV, dh, 16, length[::-1], 13)
    attend(c, rand((B, H * dh), 14))


@pytest.mark.parametrize("longest", [300, 3000])
def test_visible_nan(longest):
    """What is not finite and seen reaches the heads that see it, and no others: whole pairs and split ones."""
    c = paged(2, 4, 2, 64, 16, [40, longest], 21)
    q = rand((2, 256), 22)
    ref = c.attend(q)
    heads = lambda t: t.view(2, 4, 64)
    K, V = c.K.clone(), c.V.clone()
    for value in (float("nan"), float("inf")):
        p = q.clone()
        heads(p)[1, 3, 5] = value
        out = c.attend(p)
        assert heads(out)[1, 3].isnan().all()
        assert torch.equal(heads(out)[1, :3], heads(ref)[1, :3]) and torch.equal(out[0], ref[0])
        for row in (0, 17, longest - 1):
            pg = int(c.table[1, row // 16])
            c.K[pg, 1, row % 16] = value
            out = c.attend(q)
            c.K.copy_(K)
            if math.isnan(value):
                assert heads(out)[1, 2:].isnan().all(), row
            assert torch.equal(heads(out)[1, :2], heads(ref)[1, :2]) and torch.equal(out[0], ref[0])
            c.V[pg, 1, row % 16, 7] = value
            out = c.attend(q)
            c.V.copy_(V)
            assert not heads(out)[1, 2:, 7].isfinite().any()
    c.K[c.table[1, :-(-longest // 16)].long(), 1] = float("-inf")
    out = c.attend(q.abs())
    check()
    assert heads(out)[1, 2:].isnan().all()


@pytest.mark.parametrize("n_sink", [(1 << 31) - 16, (1 << 31) - 15, (1 << 31) - 1])
@pytest.mark.parametrize("longest", [300, 3000])
def test_more_sinks_than_rows(n_sink, longest):
    """Any number of sinks, up to the argument's last: every row is seen."""
    length = [0, 1, 17, 200, longest]
    c = paged(5, 8, 2, 64, 16, length, 23, window=20, n_sink=n_sink)
    q = rand((5, 512), 24)
    out = attend(c, q)
    c.desc.window = c.desc.n_sink = 0
    every = attend(c, q)
    assert not out[0].any() and torch.equal(out[1:3], every[1:3])


def test_results_over_the_queries():
    for longest in (300, 3000):
        c = paged(3, 4, 2, 64, 16, [40, 0, longest], 25)
        x = rand((3, 512), 26)
        ref = c.attend(x[:, :256])
        assert c.attend(x[:, :256], out=x[:, :256]).data_ptr() == x.data_ptr()
        y = rand((3, 512), 27)
        z = c.append(y[:, :256], y[:, 256:384], y[:, 384:])
        c.append(y[:, :256], y[:, 256:384], y[:, 384:], out=y[:, :256])
        with pytest.raises(pf.ProxyFormerError) as e:  # (the second sequence has no row)
            check()
        assert e.value.status == pf.PF_ERR_CAPACITY
        assert torch.equal(x[:, :256], ref) and torch.equal(y[:, :256], z)
