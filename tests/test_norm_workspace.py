"""Scratch memory of the group norm beside the size of its matrix."""
import pytest

import paper_2104_06700_amd as gnn


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("n,c,groups", [(2_400_000, 2048, 1), (2_400_000, 1025, 5), (1_000_000, 4096, 32), (500_000, 16384, 16384), (2_449_029, 1500, 3)])
def test_every_row_by_itself_needs_little_beside_the_matrix(n, c, groups, backward):
    # per statistic 8 bytes in each direction, 4 a row for its sample and 16 for a group in pieces; the rest does not grow with the rows
    rows = n * (8 * groups + 4 + 16)
    assert gnn.gnn_group_norm_workspace_bytes(n, c, groups, n, backward) - rows <= 4096 * c * 16 + 2048 * c * 8 + 4096
    assert gnn.gnn_group_norm_workspace_bytes(n, c, groups, n, backward) <= max(n * c * 2 // 4, 2 * rows)


@pytest.mark.parametrize("samples", [1, 2, 1000, 2_400_000])
def test_no_step_at_a_workgroups_width(samples):
    """From 1,024 columns to 1,025: a column more, and a group in two pieces."""
    narrow, wide = (gnn.gnn_group_norm_workspace_bytes(2_400_000, c, 1, samples, True) for c in (1024, 1025))
    assert narrow <= wide <= narrow * 1.01 + samples * 16 + 4096
