"""A dimension of a launch holds fewer than 2^32 lanes, and the runtime launches what
32 bits leave of a larger number without a word.  The calls whose kernels lie in one
dimension come back with an error there.  Run in a child process without a GPU, where
a launch that is tried fails with another message."""
import subprocess
import sys

import pytest
import torch

CHILD = """
from paper_2106_04718_amd import _native as N
A = [(i + 1) << 44 for i in range(12)]
n = {n}
st = {call}
assert st == N.FS_ERR_HIP, (st, N.last_error())
assert ("invalid configuration" in N.last_error()) == {refused}, N.last_error()
"""
CALLS = {
    "ngram": "N.lib().fs_ngram_block(A[0], 8, n, 8, 3, A[1], 4, None)",                       # 64 lanes a row
    "ancestry": "N.lib().fs_beam_ancestry_step(A[0], 1, A[1], n, 1, 0, None)",                # 256 a source
    "select": "N.lib().fs_beam_select(A[0], A[1], A[2], 8, 8, 0, A[3], A[4], A[5], n, 1, 2, 1, A[6], 1 << 40, None)",   # 512 twice
    "attention": "N.lib().fs_beam_cross_attn(A[0], A[1], A[2], A[3], A[4], n, 1, 1, 1, 16, N.FS_F32, A[5], 1 << 40, None)",
}


@pytest.mark.parametrize("name,n,refused", [
    ("ngram", 1 << 26, True), ("ngram", (1 << 26) - 1, False), ("ancestry", 1 << 24, True), ("ancestry", (1 << 24) - 1, False),
    ("select", 1 << 22, True), ("select", (1 << 22) - 1, False), ("attention", 1 << 24, True), ("attention", 1000, False)])
def test_a_launch_that_one_dimension_does_not_hold_is_refused(name, n, refused):
    if torch.cuda.is_available():
        pytest.skip("the addresses are made up: only where no launch can run")
    subprocess.run([sys.executable, "-c", CHILD.format(n=n, call=CALLS[name], refused=refused)], check=True, timeout=60)
