"""The example runs the local stream's operators together: its loss falls, and the
tokens that it serves are the rows of its forward.  Both round probabilities, rows
and the projected output to bf16 (2^-8 each)."""
import os
import subprocess
import sys

import pytest

from examples.local_attention import main

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_example():
    losses, diff = main()
    assert all(b < a for a, b in zip(losses, losses[1:])) and diff <= 4 * 2.0 ** -8


def test_sync_check_of_programs_without_them():
    """pf_sync_check reads no error word of operators that a program has not used: 8 of 12."""
    code = """
import time, torch
import paper_2608_23463_gb300 as pf
s = torch.cuda.current_stream().cuda_stream
def us(n=300):
    best = 1e9
    for _ in range(7):
        t = time.perf_counter()
        for _ in range(n):
            pf.pf_sync_check(s)
        best = min(best, (time.perf_counter() - t) / n)
    return best * 1e6
before = us()
from examples.local_attention import main
main()
print("us", before, us())
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    before, after = map(float, r.stdout.split()[-2:])
    assert before < 0.85 * after, (before, after)
