"""What the paged cache's and the sampling's entry points take, on the host alone."""
import pytest

from paper_2106_04718_amd import _native as N


def test_sampling_workspace_of_many_logits():
    """The candidates of top-k's slices are few: at most 3 KB a slice of 4096 logits."""
    for R, V in ((1, 131072), (32, 1 << 22), (32, 50264)):
        assert N.lib().fs_token_sample_workspace_bytes(R, V, N.FS_F32) <= R * (40_000 + 3 * V // 4)
