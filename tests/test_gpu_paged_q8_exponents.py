"""Attention over quantised rows whose exponents go through their whole range, against float64, and exponents of rows
that hold nothing yet.

Bar: that of the bf16 cache (tests/test_gpu_paged_chunk.py), as what the rows stand for is exact, and for results near
bf16's least numbers two things of their own: the result's own rounding, half of 2^-133, and the sums, which are of
products as small as 2^-7 of a row's value and lose half of fp32's least number (2^-150) a key each, 2^-143 of the
result's."""
import numpy as np
import pytest
import torch

from oracle import local as OL
from tests.test_gpu_local_rope import check, f64, rand
from tests.test_gpu_paged_chunk import I8, make, pools, starts

pytestmark = pytest.mark.gpu


def put_exponents(t, seed, low, high):
    """Rows' exponents low .. high in place, each as often as any other."""
    t.copy_(torch.randint(low, high + 1, t.shape, generator=torch.Generator().manual_seed(seed), dtype=I8).to("cuda"))


def compare(c, q, start, out, rows=slice(None)):
    K, V = (np.nan_to_num(t, nan=0.0) for t in pools(c))
    ref, mag = OL.paged_chunk(f64(q).reshape(q.shape[0], -1, c.dh), K, V, np.maximum(c.table.cpu().numpy(), 0), c.len.tolist(),
                              start.tolist(), c.desc.window, c.desc.n_sink)
    ref, mag, got = ref[rows], mag[rows], f64(out).reshape(ref.shape)[rows]
    assert np.isfinite(got).all()
    least = 2.0 ** -134 + 2.0 ** -143 * float(c.len.max())
    err = np.abs(got - ref) - (2.0 ** -8 * 1.01 * (mag + np.abs(ref)) + 2e-5 * mag + least)
    assert (err <= 0).all(), (err.max(), np.argwhere(err > 0)[:5])
    return ref


# (tokens, rows before them): an item that one CTA holds, pieces of few items, pieces of many
SHAPES = [(20, 0), (5, 3000), (300, 1000)]


@pytest.mark.parametrize("KV,dh", [(2, 128), (4, 64)])
@pytest.mark.parametrize("new,before", SHAPES)
@pytest.mark.parametrize("window,n_sink", [(0, 0), (40, 3)])
def test_rows_that_hold_nothing(KV, dh, new, before, window, n_sink):
    """Slots past the end, and rows that the window hides, hold any bytes and any exponent: without -128, whose rows
    are NaN as a whole, and with it."""
    c = make([before + new], 8, KV, dh, 128, 90, True, window=window, n_sink=n_sink)
    n = before + new
    seen = np.zeros(-(-n // 128) * 128, bool)
    for i in range(before, n):
        seen[:n] |= OL.visible(i, n, window, n_sink)
    start, q = starts([new]), rand((new, 8 * dh), 91, scale=1.5)
    rng = np.random.default_rng(92)
    slots = np.flatnonzero(~seen)
    at = torch.from_numpy(c.table[0].cpu().numpy()[slots // 128].astype(np.int64)).cuda(), torch.from_numpy(slots % 128).cuda()
    for low in (-127, 112, -128):
        for t in (c.K, c.V):
            t[at[0], :, at[1]] = torch.from_numpy(rng.integers(-128, 128, (len(slots), KV, dh)).astype(np.int8)).cuda()
        for t in (c.K_exp, c.V_exp):
            # each value from low on in turn, from another one on for another head
            turn = (np.arange(len(slots))[:, None] + 37 * np.arange(KV)) % (128 - low) + low
            t[at[0], :, at[1]] = torch.from_numpy(turn.astype(np.int8)).cuda()
        out = c.attend(q, start=start)
        again = c.attend(q, start=start)
        newest = c.attend(q[-1:])
        check()
        compare(c, q, start, out)
        compare(c, q[-1:], starts([1]), newest)
        assert torch.equal(out, again)


@pytest.mark.parametrize("KV,dh", [(2, 128), (4, 64), (1, 64)])
@pytest.mark.parametrize("new,before", SHAPES)
def test_exponents_of_values(KV, dh, new, before):
    """V's rows from the least numbers to the largest, both sides of what the fast conversion takes in one tile, and
    results that are all small."""
    c = make([before + new, 200], 8, KV, dh, 64, 93, True)
    start, q = starts([new, 2]), rand((new + 2, 8 * dh), 94)
    for low, high in ((-126, 104), (-3, 5), (2, 104), (-126, -110), (-126, -126), (104, 104), (-119, -118)):
        put_exponents(c.V_exp, 95, low, high)
        out = c.attend(q, start=start)
        again = c.attend(q, start=start)
        check()
        assert torch.equal(out, again)
        compare(c, q, start, out)


@pytest.mark.parametrize("KV,dh", [(2, 128), (4, 64)])
@pytest.mark.parametrize("new,before", SHAPES)
def test_exponents_of_keys(KV, dh, new, before):
    """K's rows alike.  Queries are as small as the largest keys are large, so that scores lie within some tens."""
    c = make([before + new, 200], 8, KV, dh, 64, 96, True)
    start, q0 = starts([new, 2]), rand((new + 2, 8 * dh), 97)
    for low, high in ((-10, 25), (2, 104), (-126, -120), (-126, 104), (104, 104)):
        put_exponents(c.K_exp, 98, low, high)
        # keys are normal numbers of 127 2^high at most: of 2^(high + 5) mostly
        q = q0 * 2.0 ** (-(high + 5))
        assert q.isfinite().all() and q.abs().max() > 0
        out = c.attend(q, start=start)
        again = c.attend(q, start=start)
        check()
        assert torch.equal(out, again)
        compare(c, q, start, out)


@pytest.mark.parametrize("KV,dh", [(2, 128), (4, 64)])
@pytest.mark.parametrize("new,before", SHAPES)
def test_not_finite_beside_large_exponents(KV, dh, new, before):
    """A row that is not finite, of K or of V, among rows of large exponents: who sees it gets NaN, nobody else."""
    c = make([before + new, 200], 8, KV, dh, 64, 99, True)
    start, q = starts([new, 2]), rand((new + 2, 8 * dh), 100)
    put_exponents(c.V_exp, 101, -3, 30)
    own = torch.arange(new + 2, device="cuda") < new
    for i in (0, new // 2, new - 1):
        r = before + i
        for e in (c.K_exp, c.V_exp):
            was = e.clone()
            e[int(c.table[0, r // 64]), KV - 1, r % 64] = -128
            out = c.attend(q, start=start)
            check()
            sees = own & (torch.arange(new + 2, device="cuda") >= i)
            o, g = out.view(new + 2, 8, dh), 8 // KV
            assert o[sees][:, -g:].isnan().all()
            assert o[~sees].isfinite().all() and o[:, :-g].isfinite().all()
            compare(c, q, start, torch.where(o.isnan(), 0, o).view(new + 2, -1), np.flatnonzero(~sees.cpu().numpy()))
            e.copy_(was)
