"""Blocks that share a worker's rows in the norm's gradient, as the workspace tells of them: parts * groups * cols floats, none
where up to eight blocks of a cluster add up by themselves."""
import pytest

from paper_2111_00705_b200 import binding as cd


def blocks(rows, cols, groups):
    return cd.rms_norm_workspace(rows, cols, groups) // (4 * cols)


@pytest.mark.parametrize("cols,at_once", [(768, 296), (1024, 296), (4096, 296), (8192, 148)])
@pytest.mark.parametrize("workers", [10, 12, 16])
def test_many_rows_of_several_workers_take_the_whole_gpu(workers, cols, at_once):
    got = blocks(workers * 2048, cols, workers)
    assert got == at_once // workers * workers and got > at_once * 0.9


@pytest.mark.parametrize("rows,cols,groups", [(64, 4096, 1), (500, 768, 2), (1024, 4096, 16), (2048, 4096, 16), (6144, 4096, 24), (15 * 1024, 8192, 15)])
def test_where_a_cluster_is_faster(rows, cols, groups):
    assert blocks(rows, cols, groups) == 0
