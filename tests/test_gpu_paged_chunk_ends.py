"""Attention of chunks over a paged cache whose rows behind the sequences' ends hold anything."""
import pytest
import torch

from tests.test_gpu_local_rope import check, rand
from tests.test_gpu_paged_chunk import compare, make, spoil, starts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("H,KV,dh", [(8, 2, 64), (16, 2, 128), (3, 3, 128)])
@pytest.mark.parametrize("page,new,before,window", [
    (64, [20], [0], 0), (128, [5], [3000], 0), (16, [1, 8], [100, 0], 0), (256, [300, 3], [1000, 129], 0), (48, [7, 1], [500, 40], 64),
    (128, [1, 128, 127, 129], [127, 0, 0, 0], 0)])
def test_rows_behind_the_last_token(quant, H, KV, dh, page, new, before, window):
    """What lies behind a sequence's end, NaN and infinities among it, changes no bit of any result."""
    length = [a + b for a, b in zip(new, before)]
    c = make(length, H, KV, dh, page, 70, quant, window=window, n_sink=2)
    start, q = starts(new), rand((sum(new), H * dh), 71)
    ref = c.attend(q, start=start)
    check()
    compare(c, q, start, ref)
    for value in (float("nan"), float("inf")):
        for b, n in enumerate(length):
            for r in range(n, -(-n // page) * page):
                spoil(c, int(c.table[b, r // page]), slice(None), r % page, value)
        out = c.attend(q, start=start)
        check()
        assert torch.equal(out, ref)


def median_ms(f):
    f()
    t = []
    for _ in range(5):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        f()
        b.record()
        b.synchronize()
        t.append(a.elapsed_time(b))
    return sorted(t)[2]


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("before,new", [(30000, 8), (30000, 300)])
def test_a_sequence_that_has_turned_to_nan(quant, before, new):
    """Its newest rows are NaN, those of the call's tokens among them: so are their results, and nobody waits for them.
    (A row that walks its whole cache takes 30 ms, the call without such rows 0.04 to 0.1.)"""
    c = make([before + new, 100], 16, 2, 128, 64, 72, quant)
    start, q = starts([new, 1]), rand((new + 1, 2048), 73)
    ref, ms = c.attend(q, start=start), median_ms(lambda: c.attend(q, start=start))
    for r in range(before - 10, before + new):
        spoil(c, int(c.table[0, r // 64]), slice(None), r % 64)
    out = c.attend(q, start=start)
    check()
    assert out[:new].isnan().all() and torch.equal(out[new:], ref[new:])
    late = median_ms(lambda: c.attend(q, start=start))
    print("%.3f ms, with NaN %.3f" % (ms, late))
    assert late <= 30 * ms, (ms, late)
