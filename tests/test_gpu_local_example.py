"""The example runs the local stream's operators together: its loss falls, and the
tokens that it serves are the rows of its forward.  Both round probabilities, rows
and the projected output to bf16 (2^-8 each)."""
import pytest

from examples.local_attention import main

pytestmark = pytest.mark.gpu


def test_example():
    losses, diff = main()
    assert all(b < a for a, b in zip(losses, losses[1:])) and diff <= 4 * 2.0 ** -8
