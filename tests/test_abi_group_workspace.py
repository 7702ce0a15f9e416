"""The workspace that the group norms ask for, without a GPU: by rows, features and groups, not by the number of graphs."""
import pytest


@pytest.fixture(scope="module")
def dg():
    import paper_2609_01983_amd as dg
    return dg


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("n,F,groups", [(1 << 21, 64, 32), (1 << 24, 64, 64), (1 << 21, 8192, 2048), (1 << 20, 1, 1), (123457, 128, 8)])
def test_the_number_of_graphs_does_not_count(dg, n, F, groups, backward):
    """A tile of rows has a part of two long graphs at most, whatever the number of graphs: a pair of float64 for each of the two and each group
    and 32 bytes beside, and backward as much again and two float64 for each feature and workgroup, of which there are up to 4,096 tiles' and
    as many again for graphs."""
    tiles, workgroups = 4097 + 1, 2 * (4097 + 1)
    most = tiles * (2 * 16 * groups + 32) + 1024
    if backward:
        most += tiles * 16 * groups + workgroups * 16 * F
    for graphs in (1, 1000, 1 << 16, 1 << 20, 1 << 30):
        assert dg.group_norm_workspace_bytes(n, F, groups, graphs, backward=backward) <= most, graphs
