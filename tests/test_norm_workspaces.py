"""Workspaces of the layer norm: one made for a batch holds for every smaller batch (the last one of an epoch), as those of the transforms do.
Needs no GPU."""
import pytest

from paper_2301_08527_amd import rocket


@pytest.mark.parametrize("planes,n", [(1, 3), (1, 500), (2, 500), (1, 2048), (300, 9), (1, 4100), (2, 10000), (3, 10000), (2, 20000), (1, 30000), (1, 65000), (300, 65000),
                                      (1, 140000)])
@pytest.mark.parametrize("backward", [False, True])
def test_fewer_rows_never_need_more(planes, n, backward):
    before = 0
    for rows in list(range(1, 1500)) + list(range(2000, 20000, 37)):
        need = rocket.rocket_layer_norm_workspace_bytes(rows, planes, n, backward)
        assert need >= before, rows
        before = need
