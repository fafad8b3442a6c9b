"""Windowed attention with sinks, forward and backward, against float64.  Bars: the
probabilities and their gradients are rounded to bf16 for their products (2^-8 of
the sums of absolute terms), results once more (2^-8 of themselves), the stored
output that the backward reads once; fp32 scores (64 products), exponentials and
sums keep 2e-5 of the same sums."""
import numpy as np
import pytest
import torch

import paper_2608_23463_gb300 as pf
from oracle import local as OL
from paper_2608_23463_gb300.local import PagedKVCache, QKRope, WindowAttention
from tests.test_gpu_local_rope import BF, check, f64, rand
from tests.test_local_gradients import CASES, difference, inputs

pytestmark = pytest.mark.gpu
U = 2.0 ** -8 * 1.01


def inside(name, got, ref, bar):
    got = f64(got).reshape(ref.shape)
    err = np.abs(got - ref)
    worst = (err - bar).max()
    assert np.isfinite(got).all() and worst <= 0, f"{name}: {worst:.3e} above its bar at {np.unravel_index(np.argmax(err - bar), err.shape)}"


def step(B, L, H, KV, window, n_sink, seed=1, scale=1.0):
    q, do = rand((B * L, H * 64), seed, scale=scale), rand((B * L, H * 64), seed + 1)
    k, v = rand((B * L, KV * 64), seed + 2), rand((B * L, KV * 64), seed + 3)
    op = WindowAttention(B, L, H, KV, window=window, n_sink=n_sink)
    out = op.forward(q, k, v)
    d = op.backward(q, k, v, out, do)
    check()
    s = lambda t, n: f64(t).reshape(B, L, n, 64)
    ref, mag = OL.window_fwd(s(q, H), s(k, KV), s(v, KV), window, n_sink)
    inside("out", out, ref, U * (mag + np.abs(ref)) + 2e-5 * mag)
    refs, errs = OL.window_bwd(s(q, H), s(k, KV), s(v, KV), s(do, H), window, n_sink, u=U)
    for n, a, b, e in zip(("dq", "dk", "dv"), d, refs, errs):
        # the fp32 share: 2e-5 / 2^-8 of what the roundings may do
        inside(n, a, b, e * (1 + 2e-5 / 2.0 ** -8) + U * np.abs(b) + 1e-12)
    return op, (q, k, v, do), out, d


@pytest.mark.parametrize("L", [1, 2, 127, 128, 129, 255, 256, 257, 300, 513])
@pytest.mark.parametrize("window,n_sink", [(0, 0), (1, 0), (64, 3), (200, 0), (128, 1)])
def test_lengths(L, window, n_sink):
    step(2, L, 2, 1, window, n_sink)


@pytest.mark.parametrize("window,n_sink", [
    (1, 1), (1, 700), (2, 128), (127, 127), (128, 128), (129, 129), (130, 300), (255, 5), (256, 4), (257, 256),
    (384, 4), (500, 640), (639, 1), (640, 4), (641, 4), (1 << 30, 1 << 30)])
def test_windows_and_sinks(window, n_sink):
    step(1, 641, 2, 2, window, n_sink, 5)


@pytest.mark.parametrize("B,L,H,KV", [(1, 400, 1, 1), (3, 200, 6, 2), (1, 300, 5, 1), (2, 260, 16, 1), (1, 130, 8, 8),
                                      (5, 64, 4, 2)])
def test_heads(B, L, H, KV):
    step(B, L, H, KV, 150, 20, 9)


@pytest.mark.parametrize("B,L,H,KV,window,n_sink", [(1, 2900, 12, 12, 100, 3), (1, 2500, 8, 8, 0, 0),
                                                    (2, 1700, 7, 7, 300, 140)])
def test_many_tiles(B, L, H, KV, window, n_sink):
    """Enough key tiles that only the sinks' are cut."""
    step(B, L, H, KV, window, n_sink, 13)


def test_large_scores():
    """Scores of some hundreds: the reference rises from tile to tile, rows with one key dominating.  The
    probabilities' own fp32 error grows with the score: 64 products and their sum to 2^-22 of up to 400."""
    B, L, H = 1, 500, 2
    q, k, v = rand((L, 128), 1, scale=6.0), rand((L, 128), 2, scale=6.0), rand((L, 128), 3)
    out = WindowAttention(B, L, H, H, window=200, n_sink=4).forward(q, k, v, train=False)
    check()
    s = lambda t: f64(t).reshape(B, L, H, 64)
    ref, mag = OL.window_fwd(s(q), s(k), s(v), 200, 4)
    inside("out", out, ref, U * (mag + np.abs(ref)) + 4e-4 * mag)


def test_scores_far_below_zero():
    """A row whose scores are all near -1500 is as good as any other."""
    L = 300
    q = torch.full((L, 64), 24.0, dtype=BF, device="cuda")
    k, v = rand((L, 64), 2, scale=0.01) - 8, rand((L, 64), 3)
    out = WindowAttention(1, L, 1, 1, window=130, n_sink=2).forward(q, k, v, train=False)
    check()
    s = lambda t: f64(t).reshape(1, L, 1, 64)
    ref, mag = OL.window_fwd(s(q), s(k), s(v), 130, 2)
    inside("out", out, ref, U * (mag + np.abs(ref)) + 2e-3 * mag)  # 64 products of 192, to 2^-24 of 12288 / 8 each


def test_rows_apart_in_place_of_copies():
    """Slices of one wide matrix in and out, the rest of it left alone; the same result on another stream."""
    B, L, H, KV = 2, 150, 4, 2
    op, (q, k, v, do), out, d = step(B, L, H, KV, 70, 5, 17)
    x = torch.cat((q, k, v, do), 1)
    y = torch.full((B * L, 64 * (2 * H + 2 * KV) + 8), 3.0, dtype=BF, device="cuda")
    cut = lambda t: (t[:, :256], t[:, 256:384], t[:, 384:512], t[:, 512:768])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        o = op.forward(*cut(x)[:3], out=cut(y)[3])
        op.backward(*cut(x)[:3], o, cut(x)[3], into=cut(y)[:3])
    s.synchronize()
    check()
    for a, b in zip(cut(y), d + (out,)):
        assert torch.equal(a, b)
    assert (y[:, 768:] == 3).all()


def test_repeats_bit_for_bit():
    op, (q, k, v, do), out, d = step(1, 1500, 3, 1, 90, 10, 21)
    for _ in range(3):
        o = op.forward(q, k, v)
        assert torch.equal(o, out)
        for a, b in zip(op.backward(q, k, v, o, do), d):
            assert torch.equal(a, b)


def test_sequences_do_not_meet():
    """Infinite and NaN rows of one sequence leave the others as they are."""
    B, L = 3, 200
    q, k, v, do = (rand((B * L, 128), s) for s in (1, 2, 3, 4))
    op = WindowAttention(B, L, 2, 2, window=90, n_sink=3)
    out = op.forward(q, k, v)
    d = op.backward(q, k, v, out, do)
    bad = [t.clone() for t in (q, k, v, do)]
    for t in bad:
        t[L:2 * L] = float("nan")
    bad[2][L:2 * L] = float("inf")
    out2 = op.forward(*bad[:3])
    d2 = op.backward(*bad[:3], out2, bad[3])
    check()
    for a, b in zip((out,) + d, (out2,) + d2):
        for i in (0, 2):
            assert torch.equal(a[i * L:(i + 1) * L], b[i * L:(i + 1) * L])


def test_causal():
    """Rows before a changed token stay bit for bit."""
    L = 400
    q, k, v = (rand((L, 64), s) for s in (1, 2, 3))
    op = WindowAttention(1, L, 1, 1, window=100, n_sink=3)
    a = op.forward(q, k, v, train=False)
    for t in (q, k, v):
        t[250] = -t[250] * 2
    b = op.forward(q, k, v, train=False)
    check()
    assert torch.equal(a[:250], b[:250]) and not torch.equal(a[250:], b[250:])
    assert torch.equal(a[350:], b[350:])


def test_gradients_by_differences():
    """dq, dk and dv against differences of the forward.  out is bf16 (2^-9 of about 1 a value, 64 * L of them, as a
    random sum about sqrt(64 L) 2^-9) and the step 1/4 leaves its square's share; directions add up the whole matrix."""
    L = 90
    q, k, v, do = (rand((L, 64), s) for s in (1, 2, 3, 4))
    op = WindowAttention(1, L, 1, 1, window=30, n_sink=2)
    out = op.forward(q, k, v)
    d = op.backward(q, k, v, out, do)
    h = 2.0 ** -2
    for i in range(3):
        g = rand((L, 64), 10 + i)
        x = [t.clone() for t in (q, k, v)]
        x[i] = (x[i].float() + h * g.float()).to(BF)
        y = [t.clone() for t in (q, k, v)]
        y[i] = (y[i].float() - h * g.float()).to(BF)
        move = (x[i].double() - y[i].double())
        got = ((op.forward(*x, train=False).double() - op.forward(*y, train=False).double()) * do.double()).sum()
        want = (move * d[i].double()).sum()
        norm = (move.norm() * d[i].double().norm())
        check()
        assert (got - want).abs() <= 0.1 * norm / 8 + 5 * (64 * L) ** 0.5 * 2.0 ** -8, (i, got, want, norm)


@pytest.mark.parametrize("window,n_sink", [(0, 0), (50, 4), (16, 1)])
def test_training_rows_are_the_decoded_tokens(window, n_sink):
    """Prompt and tokens one by one over the pages give the rows of the training forward: both round the
    probabilities (2^-8) and the result (2^-8) once."""
    B, L, H, KV, prompt = 2, 140, 4, 2, 77
    x = rand((B * L, (H + 2 * KV) * 64), 1)
    w = [1.0 + 0.2 * rand((64,), s, torch.float32) for s in (2, 3)]
    rope = QKRope(H, KV, 64, *w)
    q, k, v = x[:, :H * 64], x[:, H * 64:(H + KV) * 64], x[:, (H + KV) * 64:]
    qz, kz = rope.forward(q, k, L=L)
    out = WindowAttention(B, L, H, KV, window=window, n_sink=n_sink).forward(qz, kz, v, train=False).view(B, L, -1)
    c = PagedKVCache(B, H, KV, 64, 16, 2 * B * L // 16 + 2, L // 16 + 1, rope=rope, window=window, n_sink=n_sink)
    c.reserve([L] * B)
    rows = lambda t, a, b: t.view(B, L, -1)[:, a:b].reshape(B * (b - a), -1)
    start = torch.tensor([0, prompt, 2 * prompt], dtype=torch.int32, device="cuda")
    x3 = [t.contiguous() for t in (q, k, v)]
    c.advance(start)
    qp = c.append(*(rows(t, 0, prompt) for t in x3), start=start)
    assert torch.equal(qp, rows(qz, 0, prompt))
    for i in range(prompt, L):
        c.advance()
        o = c.attend(c.append(*(rows(t, i, i + 1) for t in x3)))
        mag = v.float().abs().max()
        assert ((o.float() - out[:, i].float()).abs() <= 4 * 2.0 ** -8 * mag).all()
    check()


@pytest.mark.parametrize("B,L,H,KV,window,n_sink", [(4, 640, 32, 32, 1, 0), (4, 640, 32, 4, 2, 1), (8, 130, 40, 40, 1, 0),
                                                    (3, 385, 48, 48, 129, 33)])
def test_many_short_items(B, L, H, KV, window, n_sink):
    """Several work items of a step or two on every SM: nothing runs ahead of an item that still uses its buffers."""
    step(B, L, H, KV, window, n_sink, 17)


@pytest.mark.parametrize("n_sink", [31, 32, 33, 128, 160, 161])
def test_few_sinks(n_sink):
    """The last tile of the sinks holds 32 of them at most, or more."""
    step(2, 700, 4, 2, 150, n_sink, 19)


def test_scores_of_minus_infinity():
    """A row without a finite score has no softmax: NaN, as in any row that sees one; the others stay."""
    q, k, v = rand((300, 64), 1), rand((300, 64), 2).abs() + 0.125, rand((300, 64), 3)
    op = WindowAttention(1, 300, 1, 1, window=100, n_sink=3)
    ref = op.forward(q, k, v, train=False)
    q[140] = float("-inf")
    out = op.forward(q, k, v, train=False)
    check()
    assert out[140].isnan().all()
    out[140] = ref[140]
    assert torch.equal(out, ref)


def test_results_beside_the_inputs():
    """Results in the free columns of the inputs' own rows, and none over them."""
    B, L = 2, 333
    x = rand((B * L, 12 * 64), 25)
    q, k, v, free = x[:, :256], x[:, 256:384], x[:, 384:512], x[:, 512:]
    op = WindowAttention(B, L, 4, 2, window=100, n_sink=3)
    ref = op.forward(q, k, v, train=False)
    assert op.forward(q, k, v, train=False, out=free).data_ptr() == free.data_ptr()
    check()
    assert torch.equal(free, ref)
    for out in (q, x[:, 128:384], x[:, 320:576], x[:, 64:320]):
        with pytest.raises(pf.ProxyFormerError) as e:
            op.forward(q, k, v, train=False, out=out)
        assert e.value.status == pf.PF_ERR_INVALID_ARG


def test_backward_after_refusals():
    """A refused call leaves nothing behind that a later one stumbles over."""
    q, k = rand((8, 256), 1), rand((8, 128), 2)
    rope, att = QKRope(4, 2, 64, *(rand((64,), s, torch.float32) for s in (3, 4))), WindowAttention(1, 8, 4, 2)
    out = att.forward(q, k, k)
    for bad in (q.cpu(), None, 7):
        for f in (lambda: rope.backward(bad, k, q, k), lambda: att.backward(bad, k, k, out, q)):
            with pytest.raises(pf.ProxyFormerError) as e:
                f()
            assert e.value.status == pf.PF_ERR_INVALID_ARG
    rope.backward(q, k, q, k)
    att.backward(q, k, k, out, q)
    check()


def test_what_another_stream_reads():
    """What the forward saved and the workspace are dropped while a backward on another stream still has to read them."""
    q, do = rand((3000, 256), 1), rand((3000, 256), 2)
    k, v = rand((3000, 128), 3), rand((3000, 128), 4)
    op = WindowAttention(1, 3000, 4, 2, window=200, n_sink=4)
    out = op.forward(q, k, v)
    ref = op.backward(q, k, v, out, do)
    torch.cuda.synchronize()
    side, sizes = torch.cuda.Stream(), (op.saved_size, op.ws.numel())
    fill = lambda n: torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    fill(16)  # (a first launch would wait for the other stream)
    with torch.cuda.stream(side):
        torch.cuda._sleep(1_000_000_000)  # about half a second
        d = op.backward(q, k, v, out, do)
    op.saved = op.ws = None
    junk = [fill(n) for n in sizes for _ in range(40)]
    assert not side.query()
    torch.cuda.synchronize()
    check()
    assert all(torch.equal(a, b) for a, b in zip(d, ref)) and junk


@pytest.mark.parametrize("case", CASES)
def test_gradients_along_themselves(case):
    """dq, dk and dv against differences of the forward along each of them: the bar of test_local_gradients, which
    tells a wrong sign, a wrong factor and a missing Di from the right gradient."""
    B, L, H, KV, window, n_sink = case
    op = WindowAttention(B, L, H, KV, window=window, n_sink=n_sink)
    dev = lambda t: torch.from_numpy(t).to("cuda", BF).view(B * L, -1)
    *x, do = inputs(case)
    out = op.forward(*map(dev, x))
    grads = op.backward(*map(dev, x), out, dev(do))
    check()
    forward = lambda *y: f64(op.forward(*map(dev, y), train=False)).reshape(do.shape)
    for i, d in enumerate(grads):
        got, want, bar = difference(forward, x, i, f64(d).reshape(x[i].shape), do)
        assert abs(got - want) <= bar, (i, got, want, bar)


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("L,H,KV,window,n_sink,at", [
    (300, 2, 1, 0, 0, 130), (300, 2, 1, 0, 0, 299), (300, 4, 2, 100, 3, 140), (300, 2, 2, 100, 3, 3), (300, 2, 2, 100, 3, 40),
    (700, 2, 1, 129, 40, 41), (700, 2, 1, 129, 40, 100), (700, 2, 1, 1, 0, 200), (640, 1, 1, 300, 128, 128), (77, 2, 1, 0, 0, 40)])
def test_hidden_values_do_not_matter(L, H, KV, window, n_sink, at, value):
    """A value (one column of a row of v, or all of a row of k) that is not finite reaches the rows that see it and
    no others, those of its 128-row tile among them."""
    B = 2
    q, k, v = (rand((B * L, n * 64), s) for n, s in ((H, 1), (KV, 2), (KV, 3)))
    op = WindowAttention(B, L, H, KV, window=window, n_sink=n_sink)
    s = lambda t, n: f64(t).reshape(B, L, n, 64)
    ref, mag = OL.window_fwd(s(q, H), s(k, KV), s(v, KV), window, n_sink)
    bar = U * (mag + np.abs(ref)) + 2e-5 * mag
    seen = np.array([OL.visible(i, L, window, n_sink)[at] for i in range(L)])
    assert seen[at] and not seen.all()
    for train in (False, True):
        bad = v.clone()
        bad[L + at, 7] = value  # of the first key head
        out = f64(op.forward(q, k, bad, train=train)).reshape(ref.shape)
        check()
        touched = np.zeros(ref.shape, bool)
        touched[1, seen, :H // KV, 7] = True
        assert not np.isfinite(out[touched]).any()
        assert (np.abs(out - ref)[~touched] <= bar[~touched]).all()
        bad = k.clone()
        bad[L + at, :64] = value
        out = f64(op.forward(q, bad, v, train=train)).reshape(ref.shape)
        check()
        touched = np.zeros(ref.shape, bool)
        touched[1, seen, :H // KV] = True
        assert (np.abs(out - ref)[~touched] <= bar[~touched]).all()


def test_hidden_values_in_training():
    """What a forward saved for rows before one that is not finite is theirs alone."""
    L = 300
    q, k, v, do = (rand((L, 64), s) for s in (1, 2, 3, 4))
    op = WindowAttention(1, L, 1, 1, window=100, n_sink=2)
    d = op.backward(q, k, v, op.forward(q, k, v), do)
    lse, rest = op.saved[:L * 4].clone(), op.saved[-L * 128:].view(BF).view(L, 64).clone()
    v[200] = float("nan")
    op.forward(q, k, v)
    check()
    assert torch.equal(op.saved[:200 * 4], lse[:200 * 4]) and torch.isfinite(op.saved[-L * 128:].view(BF).view(L, 64)[:200]).all()
    assert torch.isfinite(rest).all() and all(torch.isfinite(t).all() for t in d)


def test_hidden_values_of_many_items():
    """Many work items on every SM: rows that see none of the bad ones keep their values, whichever item they are of.
    Rows worked out again differ by the probabilities' rounding (2^-8 of sum p |v|, at most the largest |v|) and the
    result's."""
    B, L, H, KV, window, n_sink = 3, 1300, 40, 20, 200, 3
    q, k, v = (rand((B * L, n * 64), s) for n, s in ((H, 1), (KV, 2), (KV, 3)))
    op = WindowAttention(B, L, H, KV, window=window, n_sink=n_sink)
    ref = op.forward(q, k, v, train=False).view(B, L, H, 64)
    bad = v.clone().view(B, L, KV, 64)
    clean = torch.ones((B, L, H), dtype=torch.bool, device="cuda")
    for b, at, g in ((0, 700, 5), (0, 10, 7), (1, 1299, 0), (2, 256, 19), (2, 383, 19)):
        bad[b, at, g, 3] = float("nan")
        seen = [at <= i and (i - at < window or at < n_sink) for i in range(L)]
        clean[b, torch.tensor(seen, device="cuda"), 2 * g:2 * g + 2] = False
    out = op.forward(q, k, bad.view(B * L, -1), train=False).view(B, L, H, 64)
    check()
    assert out[..., 3][~clean].isnan().all()
    other = torch.arange(64, device="cuda") != 3
    most = 2 * U * v.float().abs().max()
    diff = (out.float() - ref.float()).abs()
    assert (diff[clean] <= most).all() and (diff[..., other] <= most).all()
    assert (diff[clean] == 0).float().mean() > 0.95  # of the others' tiles, bit for bit
