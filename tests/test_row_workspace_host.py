"""How large the workspaces of the row operators get: partial sums of as many workgroups as a launch has, no more.  No GPU needed."""
import pytest

import paper_2508_16769_amd as P

N = [1, 7, 1000, 60_000, 1_200_000, (1 << 31) - 1]


@pytest.mark.parametrize("D", [1, 32, 77, 96, 128, 1000, 1024])
def test_block(D):
    """Five sums of D columns, 768 workgroups at most and never more than rows."""
    for n in N:
        assert P.dr_block_bwd_workspace_bytes(n, D) == 4 * 5 * D * min(n, 768)


@pytest.mark.parametrize("D,F", [(1, 1), (32, 32), (64, 64), (96, 200), (128, 128), (300, 257), (1024, 1), (1, 1024), (1024, 1024)])
def test_weight_gradients(D, F):
    """256 workgroups at most, one per tile at least, each with a tile of 128 x 128 entries at most (four sums of 32 x 32, two of 32 x 64 or 64 x 64)."""
    tiles = -(-D // 128) * -(-F // 128)
    for n in N:
        assert 0 < P.dr_act8_wgrad_workspace_bytes(n, D, F) <= max(256, 2 * tiles) * 128 * 128 * 4
    assert P.dr_act8_wgrad_workspace_bytes(N[-1], 1024, 1024) == 256 * 128 * 128 * 4
