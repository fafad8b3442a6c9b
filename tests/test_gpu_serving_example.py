"""The example serves prompts in pieces: append, attention over the pages, rows read back and the windowed attention run
together.  Its rows are those of the windowed attention over the rows that the cache holds, and of a bf16 cache those
of the forward.  Both sides round probabilities, rows and the projected output to bf16 (2^-8 each)."""
import pytest
import torch

from examples.local_attention import D, LocalBlock, far, serve_in_pieces

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
@pytest.mark.parametrize("prompts,piece", [([200, 33, 320], 96), ([1, 384, 0], 500)])
def test_serving_in_pieces(dtype, prompts, piece):
    torch.manual_seed(3)
    block, x = LocalBlock(1), torch.randn(3, 384, D, device="cuda").bfloat16()
    got, held = serve_in_pieces(block, x, prompts, piece, dtype)
    assert got.isfinite().all() and far(got, held) <= 4 * 2.0 ** -8
    if dtype == torch.bfloat16:
        assert far(got, block.forward(x.view(-1, D), 384).view_as(got)) <= 4 * 2.0 ** -8
