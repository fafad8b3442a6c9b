"""Failure detection in the chunk attention, without a fault: a test hook ends the loads of every CTA after some steps,
so that the waits for the next one run out.  The call returns after one time limit (each copy that is still waited for
at the end, in a stage that it was not sent to, would add another), reports the timeout once, and the same call
afterwards gives the same bits as before."""
import pytest
import torch

import paper_2608_23463_gb300 as pf
from tests.test_gpu_local_rope import check, rand
from tests.test_gpu_paged_chunk import make, starts

pytestmark = pytest.mark.gpu
LIMIT = 50_000_000  # ns


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("KV,dh", [(2, 128), (4, 64)])
@pytest.mark.parametrize("new,before", [(8, 100000), (300, 12000)])  # items of one query tile; of two
def test_loads_that_end_early(quant, KV, dh, new, before):
    c = make([before + new], 16, KV, dh, 64, 80, quant)
    start, q = starts([new]), rand((new, 16 * dh), 81)
    ref = c.attend(q, start=start)
    check()
    for steps in (0, 1, 2, 3, 5, 8):
        try:
            pf.pf_debug_set_wait_limit_ns(LIMIT)
            pf.pf_debug_paged_chunk_steps(steps)
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            c.attend(q, start=start)
            b.record()
            with pytest.raises(pf.ProxyFormerError) as e:
                check()
        finally:
            pf.pf_debug_paged_chunk_steps(-1)
            pf.pf_debug_set_wait_limit_ns(0)
        assert e.value.status == pf.PF_ERR_TIMEOUT, str(e.value)
        # (on the device: the host may pause)
        assert 1e6 * a.elapsed_time(b) < 1.8 * LIMIT, steps
        check()  # the report cleared it
        out = c.attend(q, start=start)
        check()
        assert torch.equal(out, ref), steps
