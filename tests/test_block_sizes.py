"""Sizes that the decoder-block operators refuse."""

import paper_2608_00029_amd as cattn


def test_workspaces_of_refused_sizes():
    """None, and no overflow on the way."""
    big = (1 << 31) - 1
    for n in (big, (1 << 30) + 1):
        assert cattn.rmsnorm_bwd_workspace_bytes(n, 64) == 0 and cattn.rmsnorm_bwd_workspace_bytes(2, n) == 0
        assert cattn.swa_bwd_workspace_bytes(1, 2, 2, n, 64, 8, 2) == cattn.swa_bwd_workspace_bytes(n, 2, 2, 40, 64, 8, 2) == 0
        assert cattn.swa_bwd_workspace_bytes(1, n, n, 40, 64, 8, 2) == 0
        assert cattn.swa_decode_workspace_bytes(1, 2, 2, n, 64, 8000, 2) == cattn.swa_decode_workspace_bytes(n, 2, 2, 4096, 64, 8000) == 0
        assert cattn.swa_bwd_workspace_bytes(1, 2, 2, 1 << 20, 64, n, n) > 0  # (window and sinks are clamped to S)
    assert cattn.rmsnorm_bwd_workspace_bytes(1 << 30, 64) == 512 * 64 * 4
    assert cattn.rmsnorm_bwd_workspace_bytes(2, 60) == cattn.swa_bwd_workspace_bytes(1, 2, 2, 4096, 96, 8, 2) == 0
    assert cattn.swa_decode_workspace_bytes(1, 2, 2, 4096, 96, 4000) == 0
