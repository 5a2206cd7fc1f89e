"""Workspace of the gradients of a cell layer: only for partial sums, so none where the
rows are not split."""
import pytest

import paper_2508_06993_amd as octnca


@pytest.mark.parametrize("rows,cols,outs", [
    (8192, 4096, 4096), (16384, 8192, 8192), (1 << 20, 8192, 8192),   # as many tiles as fill the card
    (100, 1000, 500), (256, 130, 129), (0, 517, 1003),                # few rows
    (128, 32, 64), (1, 1, 1), (0, 3, 5)])                             # narrow layers
def test_none_without_splits(library_path, rows, cols, outs):
    """16 bytes: a size of 0 stands for invalid arguments."""
    assert octnca.octree_nca_mx4_backward_workspace_bytes(rows, cols, outs) == 16


@pytest.mark.parametrize("rows,cols,outs,splits", [
    (102400, 32, 64, 512), (129, 32, 64, 2), (1000, 517, 1003, 4), (257, 130, 129, 2)])
def test_partial_sums(library_path, rows, cols, outs, splits):
    assert (octnca.octree_nca_mx4_backward_workspace_bytes(rows, cols, outs) ==
            splits * outs * (cols + 1) * 4)


def test_no_size_is_too_small_for_fewer_rows(library_path):
    size = octnca.octree_nca_mx4_backward_workspace_bytes
    for cols, outs in ((1, 1), (32, 64), (129, 128), (517, 1003), (3000, 3000), (4096, 4096)):
        sizes = [size(n, cols, outs) for n in range(0, 20000, 41)]
        assert sizes == sorted(sizes)
