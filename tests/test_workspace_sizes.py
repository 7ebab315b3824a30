"""Workspace sizes of calls whose token counts differ from step to step."""
from paper_2106_04718_amd import api


def test_nothing_is_kept_for_a_number_of_tokens():
    before = len(api._WS_BYTES)
    sizes = [api.paged_chunk_attn_workspace_bytes(n, 8, 32, 8, 16, 64, 128) for n in range(1, 2000)]
    assert sizes == sorted(sizes) and sizes[0] > 0
    assert [api.paged_resize_workspace_bytes(8, n) for n in (0, 2000)] == [api.paged_resize_workspace_bytes(8, 0)] * 2
    assert len(api._WS_BYTES) == before
