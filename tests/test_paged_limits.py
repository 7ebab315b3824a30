"""What the paged cache's and the sampling's entry points take, on the host alone."""
import pytest

import pytest

from paper_2106_04718_amd import _native as N
from test_abi_paged import BIG, F, INVALID, append, attn

NEW = dict(k=7 * F, v=8 * F)


def test_sampling_workspace_of_many_logits():
    """The candidates of top-k's slices are few: at most 3 KB a slice of 4096 logits."""
    for R, V in ((1, 131072), (32, 1 << 22), (32, 50264)):
        assert N.lib().fs_token_sample_workspace_bytes(R, V, N.FS_F32) <= R * (40_000 + 3 * V // 4)


@pytest.mark.parametrize("scale", [3e38, -2.4e38])
def test_a_scale_that_overflows_in_base_2_is_refused(scale):
    """Scores are taken in base 2: with a factor of infinity a product of 0 would be NaN."""
    assert attn(scale=scale) == INVALID and "scale" in N.last_error()


@pytest.mark.parametrize("change,needle", [
    (dict(V=BIG), "one another"), (dict(ps=0), "one another"), (dict(hs=0), "one another"), (dict(ss=0), "one another"),
])
def test_a_cache_whose_slots_lie_on_one_another_is_not_written(change, needle):
    assert append(**change) == INVALID and needle in N.last_error()
    assert attn(**NEW, **change) == INVALID and needle in N.last_error()


def test_a_cache_that_is_read_alone_may_be_expanded():
    """These get as far as the workspace, which is missing."""
    for change in (dict(V=BIG), dict(ps=0), dict(hs=0), dict(ss=0), dict(ps=0, P=1, **NEW), dict(hs=0, Hkv=1, **NEW),
                   dict(ss=0, page=1, **NEW)):
        assert attn(ws=None, **change) == INVALID and "workspace" in N.last_error(), change
